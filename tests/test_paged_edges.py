"""GPU parity of the key/value cache in pages at the edges of what its entry points allow, against the float64 statements
(oracle/nova_paged.py).  Lists and means are exact; attention is held to the bounds that stand at the head of test_paged.py."""
import numpy as np
import pytest
import torch

from oracle import nova_paged as P
from paper_2602_01345_amd import PagedCache
from test_paged import DTYPES, _compare, _fill, _ints, _np, _run

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


# ---- tables with entries that are no pages ------------------------------------------------------------------------------
NONE = (-1, 2 ** 31 - 1, -2 ** 31, 1 << 20)                      # and the number of pages itself


def _choose(B, n, hk, take, pages, seed):
    g = np.random.default_rng(seed)
    return np.sort(np.stack([g.permutation(pages)[:take] for _ in range(B * n * hk)]).reshape(B, n, hk, take), axis=-1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("p", [16, 32, 64, 256])
@pytest.mark.parametrize("n,H,hk,B,take", [(1, 4, 2, 1, 0), (5, 4, 2, 1, 0), (33, 2, 2, 2, 0), (140, 4, 2, 1, 0), (5, 4, 2, 1, 3), (40, 2, 2, 1, 3),
                                           (200, 16, 16, 3, 4)])
def test_entries_that_are_no_pages_read_as_zeros_in_every_kernel(nova, dtype, dh, p, n, H, hk, B, take):
    """Blocks of 16, 32 and 128 rows, tiles of one page and of several, chosen pages in each."""
    L = max(6 * p - 9, 300)
    print(f"paged, entries that are none: {dtype} dh={dh} p={p} n={n} H={H}/{hk} B={B} take={take}", flush=True)
    cache, table = _fill(dtype, B, hk, p, dh, [L] * B, -(-L // p) + 1, 5)
    pages = -(-L // p)
    for b in range(B):
        for i in range(b % 2, pages, 2):
            table[b, i] = (*NONE, cache.k_pages.shape[0])[(i + b) % 5]
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()
    chosen = _choose(B, n, hk, take, pages, 3) if take else None
    K, V = ([P.image_rows(_np(pool), table[b], L) for b in range(B)] for pool in (cache.k_pages, cache.v_pages))
    for causal in (False, True):
        out, lse = _run(nova, cache, table, q, L, causal=causal, chosen=chosen)
        _compare(out, lse, P.attention(_np(q), K, V, dh ** -0.5, [n] * B, causal, chosen, p), dtype, dh, L)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [16, 64, 256])
@pytest.mark.parametrize("n,hk,B,take", [(1, 2, 1, 0), (5, 2, 1, 0), (140, 2, 1, 0), (5, 2, 1, 3), (200, 16, 3, 4)])
def test_pools_without_pages(nova, dtype, p, n, hk, B, take):
    """Every row is zeros: every query the mean of nothing, and the logarithm of how many rows it sees."""
    dh, L = 128, 6 * p - 9 if p > 16 else 300
    print(f"paged, no pages at all: {dtype} p={p} n={n} hk={hk} B={B} take={take}", flush=True)
    pages = -(-L // p)
    table = np.array([[(*NONE, 0)[(i + b) % 5] for i in range(pages)] for b in range(B)])
    q = torch.randn((B, n, hk, dh), generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()
    chosen = _choose(B, n, hk, take, pages, 3) if take else None
    K = [np.zeros((hk, L, dh))] * B
    out, lse = _run(nova, PagedCache.empty(0, hk, p, dh, DTYPES[dtype]), table, q, L, chosen=chosen)
    _compare(out, lse, P.attention(_np(q), K, K, dh ** -0.5, [n] * B, False, chosen, p), dtype, dh, L)


# ---- scores that are all -inf -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,H,hk,B,L,take", [(1, 2, 2, 1, 300, 4), (1, 4, 2, 2, 4000, 40), (5, 4, 2, 1, 600, 3), (40, 4, 2, 1, 900, 6),
                                             (200, 16, 16, 3, 640, 12), (200, 32, 16, 9, 640, 12)])
def test_scores_of_minus_infinity_over_chosen_pages(nova, dtype, dh, n, H, hk, B, L, take):
    """The softmax of nothing but -inf is no number, over chosen pages as over all rows; not to have chosen anything gives zeros."""
    p = 16
    print(f"paged, scores of -inf: {dtype} dh={dh} n={n} H={H}/{hk} B={B} L={L} take={take}", flush=True)
    pages = -(-L // p)
    cache, table = _fill(dtype, B, hk, p, dh, [L] * B, pages, 6)
    g = np.random.default_rng(7)
    dead = np.sort(g.permutation(pages)[:pages // 2])            # pages with keys of -inf in a channel where queries are positive
    for b in range(B):
        cache.k_pages[_ints(table[b, dead]).long(), :, :, 9] = -float("inf")
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()
    q[..., 9] = q[..., 9].abs() + 0.5
    live = np.setdiff1d(np.arange(pages), dead)
    chosen = np.full((B, n, hk, take), -1)
    kind = g.integers(0, 3, (B, n, hk))                          # nothing, dead pages alone, both
    kind[0, 0] = np.arange(hk) % 3 + 1 if n > 1 else [1, 2][:hk]
    kind = np.where(kind == 3, 0, kind)
    for at in np.ndindex(B, n, hk):
        if kind[at]:
            m = take if kind[at] == 1 else take // 2
            c = g.permutation(dead)[:m]
            chosen[at][:len(c)] = c
        if kind[at] == 2:
            c = g.permutation(live)[:take - take // 2]
            chosen[at][take - len(c):] = c
    out, lse = _run(nova, cache, table, q, L, chosen=chosen)
    K, V = ([P.image_rows(_np(pool), table[b], L) for b in range(B)] for pool in (cache.k_pages, cache.v_pages))
    for b in range(B):                                           # what a query has chosen and can weigh: the live pages
        K[b][:, np.isin(np.arange(L) // p, dead)] = 0.0
    ref = P.attention(_np(q), K, V, dh ** -0.5, [n] * B, False, np.where(np.isin(chosen, live), chosen, -1), p)
    kind = kind.repeat(H // hk, 2)
    got, glse = _np(out), _np(lse)
    assert np.isnan(got[kind == 1]).all() and np.isneginf(glse[kind == 1]).all() and (kind == 1).any()
    nan = torch.from_numpy(kind == 1).cuda()
    out[nan] = 0.0
    _compare(out, lse, ref, dtype, dh, L)
    # over all rows, where nothing else is
    for b in range(B):
        cache.k_pages[_ints(table[b]).long(), :, :, 9] = -float("inf")
    out, lse = _run(nova, cache, table, q, L)
    assert torch.isnan(out).all() and torch.isneginf(lse).all()


# ---- divisions of large calls ---------------------------------------------------------------------------------------------
def _check_some(nova, B, H, hk, dh, p, n, kv_len, lens=None, counts=None, causal=False, take=0, seed=1, dtype="bf16"):
    """A large call, held against the oracle at some queries of every image: the first and last row of blocks of 128 rows, the last live
    one, some others.  What has no query is zeros."""
    print(f"paged attention, large: B={B} H={H}/{hk} dh={dh} p={p} n={n} kv_len={kv_len} lens={lens} counts={counts} causal={causal} "
          f"take={take}", flush=True)
    real, live = lens or [kv_len] * B, counts or [n] * B
    cache, table = _fill(dtype, B, hk, p, dh, real, -(-kv_len // p), seed)
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(seed)).to(DTYPES[dtype]).cuda()
    g = np.random.default_rng(seed)
    chosen = None
    if take:
        pages = -(-kv_len // p)
        chosen = np.sort(np.argpartition(g.random((B, n, hk, pages), dtype=np.float32), take - 1)[..., :take], axis=-1)
    out, lse = _run(nova, cache, table, q, kv_len, lens, counts, causal, None, chosen)
    assert torch.isfinite(out).all()
    G, pools, queries = H // hk, [_np(cache.k_pages), _np(cache.v_pages)], _np(q)
    for b in range(B):
        assert (out[b, live[b]:] == 0).all() and torch.isneginf(lse[b, live[b]:]).all()
        rows = {0, n * G - 1, live[b] * G - 1, *(128 * g.integers(0, n * G // 128, 3)), *(128 * g.integers(1, n * G // 128, 3) - 1), *g.integers(0, n * G, 4)}
        for row in sorted(int(r) for r in rows if r >= 0):
            s, h = row // G, int(g.integers(0, hk)) * G + row % G
            sees = int(P.visible(real[b], live[b], n, causal)[s])
            K, V = ([P.image_rows(pool[:, h // G:h // G + 1], table[b], real[b])[:, :sees]] for pool in pools)
            one = None if chosen is None else chosen[b:b + 1, s:s + 1, h // G:h // G + 1]
            ref = P.attention(queries[b:b + 1, s:s + 1, h:h + 1], K, V, dh ** -0.5, [1 if s < live[b] else 0], False, one, p)
            _compare(out[b:b + 1, s:s + 1, h:h + 1], lse[b:b + 1, s:s + 1, h:h + 1], ref, dtype, dh, kv_len)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,H,hk,n,kv_len,lens,counts", [(1, 16, 16, 2170, 4100, None, None), (2, 8, 8, 2170, 4100, [4100, 2200], None),
                                                         (3, 32, 4, 400, 4200, [400, 4200, 90], [400, 350, 90]), (2, 10, 10, 2000, 4160, [100, 4160], [0, 1999])])
def test_a_few_more_items_than_cus_in_three_runs(nova, B, H, hk, n, kv_len, lens, counts, causal):
    """257 to 320 blocks of 128 rows with heads of 128 over 64 tiles or more; images of which some runs have nothing."""
    assert 256 < B * hk * -(-n * (H // hk) // 128) <= 320
    _check_some(nova, B, H, hk, 128, 64, n, kv_len, lens, counts, causal)


@pytest.mark.parametrize("H,hk,n,pages,take", [(16, 16, 2150, 300, 20), (32, 8, 1080, 512, 16)])
def test_chosen_pages_in_three_runs(nova, H, hk, n, pages, take):
    assert 256 < hk * -(-n * (H // hk) // 128) <= 320
    _check_some(nova, 1, H, hk, 128, 16, n, pages * 16 - 3, take=take, causal=True)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,hk,n,kv_len", [(4, 16, 2100, 2200), (9, 16, 500, 700), (32, 4, 1020, 1100), (5, 30, 520, 900)])
def test_images_by_falling_length(nova, dh, B, hk, n, kv_len):
    """More blocks than two rounds of the chip, none of them cut, and fewer, of which the last are; images of every length."""
    assert B * hk * -(-n // 128) > 512
    g = np.random.default_rng(B)
    lens = [int(x) for x in g.integers(1, kv_len + 1, B)]
    lens[1], lens[-1] = kv_len, 0
    _check_some(nova, B, hk, hk, dh, 32, n, kv_len, lens, [min(n, x) for x in lens], causal=True)
    _check_some(nova, B, hk, hk, dh, 32, n, kv_len, lens, None)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("pages", [720, 732, 736, 900])
def test_lists_about_what_leaves_room_for_a_second_workgroup(nova, dh, pages):
    _check_some(nova, 1, 16, 16, dh, 16, 600, pages * 16 - 5, take=16, causal=True)


# ---- means ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_largest_numbers_just_above_127_units(nova, dtype):
    """127.25 takes a unit of 2, in means and in queries: a page of 100 beats one whose product with 127 would have won."""
    rows = torch.zeros((2, 1, 16, 64))
    rows[0, 0, ::2, 0], rows[0, 0, 1::2, 0], rows[0, 0, :, 1] = 127.0, 127.5, 3.0           # 127.25 on average
    cache = PagedCache(*[rows.to(DTYPES[dtype]).cuda() for _ in range(2)])
    means = torch.zeros((2, 1, 64), dtype=torch.bfloat16, device="cuda")
    nova.paged_summarise(cache, _ints([[0, 1]]), means, 32, 32)
    assert means[0, 0, :2].tolist() == [128.0, 4.0]
    m = torch.zeros((2, 1, 64), dtype=torch.bfloat16, device="cuda")
    m[0, 0, 0], m[1, 0, 1] = 1.0, 100.0
    for scale in (1.0, 2.0 ** -9, 2.0 ** 40):
        q = torch.zeros((1, 2, 1, 64))
        q[0, 0, 0, :2], q[0, 1, 0, :2] = torch.tensor([127.25 if dtype == "f32" else 127.5, 1.4]) * scale, torch.tensor([126.5, 1.0]) * scale
        q = q.to(DTYPES[dtype]).cuda()
        chosen = torch.empty((1, 2, 1, 1), dtype=torch.int32, device="cuda")
        nova.paged_select(m, _ints([[0, 1]]), 16, q, chosen, 32, first=0, recent=0)
        assert np.array_equal(chosen.cpu().numpy(), P.select(_np(q), _np(m), np.array([[0, 1]]), 16, [32], [2], False, 0, 0, 1))
        assert chosen.flatten().tolist() == [1, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p,keep", [(16, 37), (16, 32), (64, 1), (256, 300), (32, 0)])
def test_means_of_images_that_were_cut_back(nova, dtype, p, keep):
    """Without rows to come the last page's mean is the old one until it is asked for; other pages' never change."""
    hk, dh, L = 2, 64, 310
    cache, table = _fill(dtype, 1, hk, p, dh, [L], -(-L // p), 2)
    tt, lens, count = _ints(table), _ints([L]), _ints([0])
    means = torch.zeros((cache.k_pages.shape[0], hk, dh), dtype=torch.bfloat16, device="cuda")
    nova.paged_summarise(cache, tt, means, L, L)
    before = _np(means)
    nova.paged_reserve(tt, p, 0, L, torch.zeros(cache.k_pages.shape[0], dtype=torch.int32, device="cuda"), count, lens, kv_len_per_row=lens,
                       keep_per_row=_ints([keep]))
    assert lens.item() == keep
    nova.paged_summarise(cache, tt, means, 1, L, n_per_row=_ints([0]), kv_len_per_row=lens)
    assert np.array_equal(_np(means), before)
    nova.paged_summarise(cache, tt, means, 1, L, kv_len_per_row=lens)
    want = P.summarise(_np(cache.k_pages), table, before, [keep], [1])
    assert np.array_equal(_np(means), want) and np.array_equal(want, before) == (keep % p == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
def test_rows_copied_within_the_pools(nova, dtype, dh):
    """An image's last page written once more for another that begins alike: the sources are rows of the pools, no slot is one of them."""
    p, hk, L = 32, 3, 80
    cache, table = _fill(dtype, 1, hk, p, dh, [L], 3, 2)
    before = [_np(t) for t in (cache.k_pages, cache.v_pages)]
    last, spare = int(table[0, 2]), next(i for i in range(cache.k_pages.shape[0]) if i not in table)
    slots = np.array([[spare * p + r for r in range(L - 2 * p)]])
    k, v = (t[last:last + 1, :, :L - 2 * p].transpose(1, 2) for t in (cache.k_pages, cache.v_pages))
    rows = [_np(k), _np(v)]
    nova.paged_append(cache, k, v, _ints(slots))
    for t, was, new in zip((cache.k_pages, cache.v_pages), before, rows):
        assert np.array_equal(_np(t), P.append(was, new, slots), equal_nan=True)
