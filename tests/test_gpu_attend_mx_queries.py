"""fp32 queries of 17 to 32 rows over short 4-bit caches: their three terms lie where the waves'
sums are put afterwards, beside kept logits, in many workgroups at once."""
import pytest

from attend_more import run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(17, 1), (5, 4), (3, 7), (8, 4)])
@pytest.mark.parametrize("N", [1, 31, 129, 256, 500])
def test_queries_beside_kept_logits(N, T, G, D):
    run_case(70, 8, G, D, T, N, N + 3, "fp32", True)
    run_case(9, 2, G, D, T, N, N + 3, "fp32", True, lens=[N, 0, 1, N // 2, 7, 64, N, 3, N - 1], causal=False)
    run_case(9, 2, G, D, T, N, N + 3, "fp32", True, window=N // 2 + 1, sinks=3)
