"""The contractions' DRAM traffic in the benchmark's line: read from the committed counters, which name the sources that
they were taken of."""
import bench
from paper_2606_19528_gb300 import workloads


def test_counters_are_those_of_the_present_sources():
    wl = workloads.llama_layer_T2048()
    # W, x and dy once, y and dx once, in bf16: 808 MB; the tiles' walk reads a little less (L2) to a tenth more
    assert 0.9 * 808e6 < bench.gemm_traffic(wl.name) < 1.1 * 808e6
    assert bench.gemm_traffic("another") is None
