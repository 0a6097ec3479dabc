"""Host-only: the rocprofv3 figures that the benchmark cites are of the kernel sources in this tree."""
import bench


def test_recorded_for_these_sources():
    with open(bench.RECORDED) as f:
        kernel = next(l.split("=", 1)[1].strip() for l in f if l.startswith("kernel ="))
    rec, why_not = bench.recorded_counters("cfg2", kernel)
    assert rec is not None, why_not
    assert float(rec["rocprof_avg_ns"]) > 0 and float(rec["fetch_size_kib"]) > 0 and float(rec["write_size_kib"]) > 0
