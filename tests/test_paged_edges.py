"""GPU parity of the key/value cache in pages at the edges of what its entry points allow, against the float64 statements
(oracle/nova_paged.py).  Lists and means are exact; attention is held to the bounds that stand at the head of test_paged.py."""
import numpy as np
import pytest
import torch

from oracle import nova_paged as P
from test_paged import _ints, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nova():
    import harness
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU and the built libnova.so (no fallback)")
    return harness.nova()


# ---- which pages a query chooses --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pages,k,first,recent", [(8, 3, 1, 1), (8, 2, 0, 2), (60, 12, 3, 4), (300, 20, 1, 1), (300, 256, 100, 100), (700, 9, 9, 0),
                                                  (1500, 40, 1, 7), (5000, 64, 1, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_pages_of_nan_take_no_place_of_first_and_recent_ones(nova, dtype, pages, k, first, recent, causal):
    """More pages with means of NaN than there are places: `first` and `recent` pages are chosen all the same."""
    if causal and recent == 0:
        first, recent = first - 1, 1
    print(f"paged select, means of NaN: pages={pages} k={k} {first}/{recent} causal={causal} {dtype}", flush=True)
    p, hk, H, dh, n = 16, 2, 6, 64, 5
    g = np.random.default_rng(pages)
    m = np.array([[P.seven_bits(x) for x in page] for page in g.standard_normal((pages, hk, dh))])
    odd = g.permutation(pages)[:max(pages // 2, k)]
    m[odd, 0] = np.nan
    m[odd[:k // 2], 1] = np.nan
    table = g.permutation(pages)[None]
    q = torch.randn((1, n, H, dh), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    chosen = torch.full((1, n, hk, k), -99, dtype=torch.int32, device="cuda")
    L = pages * p - 3
    nova.paged_select(torch.from_numpy(m).to(torch.bfloat16).cuda(), _ints(table), p, q, chosen, L, first=first, recent=recent, causal=causal)
    got = chosen.cpu().numpy()
    assert np.array_equal(got, P.select(_np(q), m, table, p, [L], [n], causal, first, recent, k))
    for s in range(n):
        sees = -(-(L - n + s + 1 if causal else L) // p)
        for j in range(hk):
            assert set(range(first)) | set(range(max(sees - recent, 0), sees)) <= set(got[0, s, j].tolist())
