"""GPU parity of the 4-bit key/value cache with its float64 statements (oracle/nova_fourbit.py).

Tolerances, element by element.  Codes, scales and moved rows are exact.  With u = 2^-24 (fp32), S the largest
sum_c |q_c k_c| * scale of a query and L keys, a score is a sum of dh products and a factor, off by at most (dh + 8) u S, and
2^x adds 4 u and the rounding of its argument, 2 u (S + |lse|); so every probability is off by d = (2 dh + 32) u (S + |lse| + 1)
of itself (numerator and sum), and a sum over L of them is taken in chains of at most L / 2 + 64 roundings.
  out   d_out = (2 d + (L + 128) u) w with w = sum_j p_j |v_j|; bf16: probabilities and results are rounded once each, half a
        step is 2^-8: + 2^-8 w + 2^-8 |out|, and 2 % for products of the two.  fp32 ends at 2^-126: a term e^(s - max) v, its
        factor or its rescaling below that may become 0, at most 4 * 2^-126 (1 + |v|) each, L of them
  lse   d + (L + 128) u + 8 u |lse|
  mass  what is collected times (2 d + (n heads + 128) u), + 2 u mass"""
import numpy as np
import pytest
import torch

from oracle import nova_fourbit as F
from paper_2602_01345_amd import FourBitCache

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def nova():
    import harness
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU and the built libnova.so (no fallback)")
    return harness.nova()


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _ints(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device="cuda")


def _fill(B, hk, cap, dh, lens, seed, scale=1.0, dead=255):
    """A cache with rows [0, lens[b]), everything behind them `dead`; and its halves for the oracle."""
    g = np.random.default_rng(seed)
    halves = []
    for _ in range(2):
        x = (scale * g.standard_normal((B, hk, cap, dh)) * np.exp(0.5 * g.standard_normal((hk, 1, dh)))).astype(np.float32)
        codes, scales = F.quantise(x)
        for b, n in enumerate(lens):
            codes[b, :, n:], scales[b, :, n:] = dead, dead
        halves.append((codes, scales))
    return FourBitCache(*[torch.from_numpy(t).cuda() for h in halves for t in h]), halves


def _fill_codes(B, hk, cap, dh, lens, seed, scale=1.0, dead=255):
    """The same of any codes, for large caches: quantising on the host takes its time."""
    g = np.random.default_rng(seed)
    halves = []
    for _ in range(2):
        codes = g.integers(0, 256, (B, hk, cap, dh // 2), dtype=np.uint8)
        scales = g.integers(124, 127, (B, hk, cap, dh // 32), dtype=np.uint8)
        for b, n in enumerate(lens):
            codes[b, :, n:], scales[b, :, n:] = dead, dead
        halves.append((codes, scales))
    return FourBitCache(*[torch.from_numpy(t).cuda() for h in halves for t in h]), halves


def _values(half, lens):
    v = F.values(*half)
    for b, n in enumerate(lens):
        v[b, :, n:] = 0.0
    return v


def _bounds(ref, dtype, dh, L, vmax=2.0 ** 20):
    out, lse, w, reach = ref
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    d = (2 * dh + 32) * U * (reach + finite + 1)
    t = (2 * d + (L + 128) * U)[..., None] * w + L * 4 * 2.0 ** -126 * (1 + vmax)
    if dtype == "bf16":
        t = t + 1.02 * 2.0 ** -8 * (w + np.abs(out))
    return t, d + (L + 128) * U + 8 * U * finite, d


def _run_attention(nova, cache, q, kv_len, lens=None, counts=None, scale=None):
    B, n, H, dh = q.shape
    need = nova.fourbit_attention_workspace_bytes(cache, H, n, kv_len)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")       # NaN wherever it is read before it is written
    out = torch.full((B, n, H, dh), float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full((B, n, H), float("nan"), device="cuda")
    nova.fourbit_attention(cache, q, out, ws, kv_len, scale=scale, lse=lse, n_per_row=counts, kv_len_per_row=lens)
    torch.cuda.synchronize()
    return out, lse


def _check_attention(nova, dtype, B, H, hk, dh, n, cap, kv_len, lens=None, counts=None, scale=None, seed=1, kscale=1.0, q=None, fill=_fill):
    print(f"fourbit attention {dtype} B={B} H={H}/{hk} dh={dh} n={n} kv_len={kv_len} lens={lens} counts={counts}", flush=True)
    real = [kv_len] * B if lens is None else [min(max(x, 0), kv_len) for x in lens]
    live = [n] * B if counts is None else [min(max(x, 0), n) for x in counts]
    cache, halves = fill(B, hk, cap, dh, real, seed, kscale)
    if q is None:
        q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(seed)).to(DTYPES[dtype]).cuda()
    out, lse = _run_attention(nova, cache, q, kv_len, None if lens is None else _ints(lens), None if counts is None else _ints(counts),
                              scale)
    sc = dh ** -0.5 if scale is None else scale
    ref = F.attention(_np(q), _values(halves[0], real), _values(halves[1], real), sc, real, live)
    t_out, t_lse, d = _bounds(ref, dtype, dh, kv_len)
    got, glse = _np(out), _np(lse)
    empty = np.isneginf(ref[1])
    assert np.array_equal(np.isneginf(glse), empty)
    assert (got[empty] == 0).all()
    assert np.isfinite(got).all()
    bad = np.abs(got - ref[0]) > t_out
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - ref[0]).max(), t_out[bad][:4])
    with np.errstate(invalid="ignore"):
        assert (np.where(empty, 0.0, np.abs(glse - ref[1])) <= t_lse).all()
    # what the rows collect from these queries
    need = nova.fourbit_mass_workspace_bytes(cache, H, n, kv_len)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    m_in = torch.rand((B, cap), generator=torch.Generator().manual_seed(seed + 1)).cuda()
    m_in[:, ::3] = -1.0
    m_in[:, 1::7] = float("nan")
    mass = torch.full((B, cap), float("nan"), device="cuda")
    l64 = ref[1].copy()
    lse_in = torch.from_numpy(l64.astype(np.float32)).cuda()
    nova.fourbit_mass(cache, q, lse_in, mass, ws, kv_len, scale=scale, mass_in=m_in,
                      n_per_row=None if counts is None else _ints(counts), kv_len_per_row=None if lens is None else _ints(lens))
    ref_m, got_m = F.mass(_np(q), _values(halves[0], real), sc, _np(lse_in), _np(m_in), real, live)
    most = d.max() if d.size else 0.0
    tol = got_m * (2 * most + (n * H + 128) * U) + 2 * U * np.abs(ref_m) + 1e-30
    diff = np.abs(_np(mass) - ref_m)
    assert (diff <= tol).all(), (np.argwhere(~(diff <= tol))[:4], diff.max())
    for b in range(B):
        assert (mass[b, real[b]:] == -1).all()
    return out, lse


# ---- append, unpack -------------------------------------------------------------------------------------------------
def _sources(B, n, hk, dh, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, n, 3 * hk, dh), generator=g) * torch.exp(2 * torch.randn((1, 1, 3 * hk, 1), generator=g))
    joint = x.to(DTYPES[dtype]).cuda()
    k, v = joint[:, :, hk:2 * hk], joint[:, :, 2 * hk:]
    pad = torch.full((B, hk, n + 3, dh), 7.0, dtype=DTYPES[dtype], device="cuda")
    padv = torch.full((B, hk, dh, n + 5), 7.0, dtype=DTYPES[dtype], device="cuda")
    pad[:, :, 1:n + 1] = k.permute(0, 2, 1, 3)
    padv[:, :, :, 3:n + 3] = v.permute(0, 2, 3, 1)
    odd = torch.full((B, n, hk, dh + 1), 7.0, dtype=DTYPES[dtype], device="cuda")     # rows that no vector load can take
    odd[..., 1:] = k
    return {"joint": (k, v), "rows": (k.contiguous(), v.contiguous()), "odd": (odd[..., 1:], v.contiguous()),
            "caches": (pad[:, :, 1:n + 1].permute(0, 2, 1, 3), padv[..., 3:n + 3].permute(0, 3, 1, 2))}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,hk,n,P", [(1, 1, 1, 0), (3, 5, 1, 37), (2, 3, 70, 9), (1, 2, 257, 300)])
def test_append_is_exact_and_touches_nothing_else(nova, dtype, dh, B, hk, n, P):
    cap = P + n + 2
    lens = [max(P - 5 * b, 0) for b in range(B)]
    counts = [n if b == 0 else n // (b + 1) for b in range(B)]
    for name, (k, v) in _sources(B, n, hk, dh, dtype, 11).items():
        print(f"fourbit append {dtype} dh={dh} B={B} hk={hk} n={n} P={P} {name}", flush=True)
        for lv, cv in ((None, None), (lens, counts)):
            cache, halves = _fill(B, hk, cap, dh, [cap] * B, 5)
            nxt = torch.full((B,), -7, dtype=torch.int32, device="cuda")
            nova.fourbit_append(cache, k, v, P, n_per_row=None if cv is None else _ints(cv),
                                kv_len_per_row=None if lv is None else _ints(lv), kv_len_next=nxt)
            lr, cr = lv or [P] * B, cv or [n] * B
            assert nxt.tolist() == [a + c for a, c in zip(lr, cr)]
            for x, half, got in ((k, halves[0], (cache.k_codes, cache.k_scales)), (v, halves[1], (cache.v_codes, cache.v_scales))):
                codes, scales = F.quantise(_np(x).transpose(0, 2, 1, 3))
                want = [half[0].copy(), half[1].copy()]
                for b in range(B):
                    want[0][b, :, lr[b]:lr[b] + cr[b]] = codes[b, :, :cr[b]]
                    want[1][b, :, lr[b]:lr[b] + cr[b]] = scales[b, :, :cr[b]]
                assert np.array_equal(got[1].cpu().numpy(), want[1]) and np.array_equal(got[0].cpu().numpy(), want[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("source", ["joint", "caches"])
def test_append_at_the_ends_of_the_range(nova, dtype, source):
    """Zeros, ties, the smallest and the largest numbers, NaN and infinities."""
    big = 3.0e38
    rows = np.zeros((1, 9, 1, 64), dtype=np.float32)
    rows[0, 0, 0, :8] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5]
    rows[0, 1, 0, :] = 1e-39
    rows[0, 2, 0, :3] = [big, -big, big / 8]
    rows[0, 3, 0, 5] = np.nan
    rows[0, 4, 0, 40] = np.inf
    rows[0, 5, 0, 63] = -np.inf
    rows[0, 6, 0, :4] = [-0.0, -1e-30, 6, -0.2]
    rows[0, 7, 0, :2] = [2.0 ** -121, 2.0 ** -125]
    t = torch.from_numpy(rows).to(DTYPES[dtype]).cuda()
    if source == "caches":
        t = t.permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2)
    cache = FourBitCache.empty(1, 1, 9, 64)
    nova.fourbit_append(cache, t, t, 0)
    x = t.to(torch.float64).cpu().numpy().transpose(0, 2, 1, 3)
    codes, scales = F.quantise(x)
    assert np.array_equal(cache.k_scales.cpu().numpy(), scales) and np.array_equal(cache.k_codes.cpu().numpy(), codes)
    assert torch.equal(cache.k_codes, cache.v_codes) and torch.equal(cache.k_scales, cache.v_scales)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,hk,n,first", [(1, 1, 1, 0), (2, 3, 65, 7), (3, 1, 130, 20)])
def test_unpack(nova, dtype, dh, B, hk, n, first):
    cap = first + n + 1
    cache, halves = _fill(B, hk, cap, dh, [cap] * B, 9)
    cache.k_scales[0, 0, first, 0] = 255                         # one group that reads as NaN
    halves[0][1][0, 0, first, 0] = 255
    firsts, counts = [max(first - 3 * b, 0) for b in range(B)], [n // (b + 1) for b in range(B)]
    for layout, (k, v) in _sources(B, n, hk, dh, dtype, 12).items():
        print(f"fourbit unpack {dtype} dh={dh} B={B} hk={hk} n={n} {layout}", flush=True)
        for fv, cv in ((None, None), (firsts, counts)):
            nova.fourbit_unpack(cache, first, k, v, first_per_row=None if fv is None else _ints(fv),
                                n_per_row=None if cv is None else _ints(cv))
            for t, half in ((k, halves[0]), (v, halves[1])):
                val = F.values(*half).transpose(0, 2, 1, 3)
                want = np.zeros((B, n, hk, dh))
                for b in range(B):
                    f, c = (fv or [first] * B)[b], (cv or [n] * B)[b]
                    want[b, :c] = val[b, f:f + c]
                assert np.array_equal(_np(t), want, equal_nan=True)
    only = torch.empty((B, n, hk, dh), dtype=DTYPES[dtype], device="cuda")
    nova.fourbit_unpack(cache, first, None, only)
    assert np.array_equal(_np(only), F.values(*halves[1]).transpose(0, 2, 1, 3)[:, first:first + n])


def test_unpack_leaves_what_lies_between_the_rows(nova):
    cache, _ = _fill(1, 2, 40, 64, [40], 3)
    pad = torch.full((1, 2, 70, 64), 7.0, device="cuda")
    nova.fourbit_unpack(cache, 0, pad[:, :, 10:50].permute(0, 2, 1, 3), None)
    assert (pad[:, :, :10] == 7).all() and (pad[:, :, 50:] == 7).all() and not (pad[:, :, 10:50] == 7).any()


# ---- attention and mass ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,L", [(1, 1), (1, 15), (1, 16), (1, 17), (1, 31), (1, 33), (1, 64), (1, 129), (1, 700), (1, 3001),
                                 (2, 5), (7, 63), (16, 65), (17, 64), (31, 200), (33, 127), (64, 640), (127, 96), (129, 1),
                                 (130, 259), (300, 1030)])
def test_lengths(nova, dtype, dh, n, L):
    _check_attention(nova, dtype, 2, 2, 2, dh, n, L + 3, L)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,hk", [(1, 1), (6, 2), (8, 1), (12, 4), (32, 2), (40, 1)])
@pytest.mark.parametrize("n,L", [(1, 300), (3, 77), (50, 190)])
def test_shared_key_heads(nova, dtype, dh, H, hk, n, L):
    _check_attention(nova, dtype, 2, H, hk, dh, n, L, L)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,kv_len", [(1, 40), (1, 2000), (9, 300), (40, 700), (200, 500), (1, 0), (150, 0)])
def test_images_with_their_own_lengths(nova, dtype, dh, n, kv_len):
    """No rows, one row, counts past either bound (clamped), images without queries; NaN behind every length."""
    lens = [kv_len, 0, 1, kv_len // 2, kv_len + 9, -3]
    counts = [n, n, n + 5, 0, max(n - 1, 0), n]
    _check_attention(nova, dtype, 6, 4, 2, dh, n, kv_len + 70, kv_len, lens, counts)
    _check_attention(nova, dtype, 6, 4, 2, dh, n, kv_len + 70, kv_len, lens, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,L", [(33, 2049), (128, 2112), (129, 2111), (300, 2113), (257, 4100)])
def test_blocks_of_128_rows_over_many_tiles(nova, dtype, dh, n, L):
    """Too many tiles for blocks of 32 rows: ends of tiles and blocks of the kernel for many rows, in runs of keys."""
    _check_attention(nova, dtype, 1, 2, 1, dh, n, L + 1, L)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,L", [(70, 1), (65, 63), (33, 64), (96, 65), (70, 129), (130, 200)])
def test_blocks_of_128_rows_of_many_heads(nova, dtype, dh, n, L):
    """Too many key heads for blocks of 32 rows: the same kernel with a tile or a few, whole items only."""
    _check_attention(nova, dtype, 9, 30, 30, dh, n, L, L)
    _check_attention(nova, dtype, 9, 30, 30, dh, n, L, L, lens=[L - b * L // 9 for b in range(8)] + [0], counts=[n - 3 * b for b in range(9)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [None, [700, 699, 0, 64, 1, 333, 650, 128, 700]])
def test_whole_items_and_runs_in_one_launch(nova, dtype, lens):
    """More blocks of queries than there is room for at a time: a full round of whole ones, the rest cut into runs of keys."""
    _check_attention(nova, dtype, 9, 32, 32, 64, 140, 700, 700, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,hk,n", [(2, 150, 130), (2, 520, 40), (31, 18, 40), (32, 33, 40), (33, 33, 40)])
def test_many_items_of_images_in_any_order(nova, dtype, dh, B, hk, n):
    """More blocks of queries than there is room for, of few and of many images: those come by length, or as they are; lengths of
    zero, past the bound and alike, images with fewer queries."""
    L = 140
    lens = [(b * 97 + 40) % (L + 20) if b % 5 else (0, L, 64, L + 9)[b // 5 % 4] for b in range(B)]
    counts = [n if b % 3 else n - 2 * b for b in range(B)]
    _check_attention(nova, dtype, B, hk, hk, dh, n, L + 1, L, lens=lens[::-1], counts=counts, fill=_fill_codes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
def test_a_few_more_blocks_than_fit_at_once(nova, dtype, dh):
    """Cut into three runs, of which some have no keys."""
    _check_attention(nova, dtype, 4, 65, 65, dh, 33, 4033, 4033, lens=[4033, 65, 0, 129], fill=_fill_codes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,H,hk,L", [(511, 1, 1, 130), (512, 2, 2, 257), (513, 1, 1, 64), (545, 2, 2, 1), (86, 12, 2, 300), (1100, 2, 1, 255)])
def test_weights_from_hundreds_of_rows(nova, dtype, dh, n, H, hk, L):
    """Around the size from which a tile has 64 rows: ends inside either half of one, heads that change inside it, runs that get
    none, images with fewer rows than that."""
    _check_attention(nova, dtype, 1, H, hk, dh, n, L + 2, L)
    _check_attention(nova, dtype, 4, H, hk, dh, n, L + 2, L, lens=[L, L // 2, 0, L], counts=[n, n - 33, n, 3])


def test_no_queries_leave_the_weights_as_they_were(nova):
    cache, _ = _fill(2, 2, 30, 64, [30, 30], 1)
    q = torch.empty((2, 0, 4, 64), dtype=torch.bfloat16, device="cuda")
    m = torch.rand((2, 30), device="cuda")
    m[0, 3], m[1, 4] = -1.0, float("inf")
    out = torch.empty_like(m)
    nova.fourbit_mass(cache, q, torch.empty((2, 0, 4), device="cuda"), out, None, 20, mass_in=m, kv_len_per_row=_ints([20, 7]))
    want = torch.where(m > 0, m, 0.0)
    want[0, 20:], want[1, 7:] = -1.0, -1.0
    assert torch.equal(out, want)
    nova.fourbit_attention(cache, q, torch.empty_like(q), None, 20)


@pytest.mark.parametrize("n", [1, 40])
def test_weights_of_protected_rows_stay_infinite(nova, n):
    cache, _ = _fill(1, 2, 90, 64, [90], 1)
    q = torch.randn((1, n, 2, 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    ws = torch.empty(max(nova.fourbit_mass_workspace_bytes(cache, 2, n, 90), 16), dtype=torch.uint8, device="cuda")
    out, lse = _run_attention(nova, cache, q, 90)
    m = torch.zeros((1, 90), device="cuda")
    m[0, 70:] = float("inf")
    nova.fourbit_mass(cache, q, lse, m, ws, 90, mass_in=m)                        # in place
    assert torch.isinf(m[0, 70:]).all() and torch.isfinite(m[0, :70]).all() and (m[0, :70] > 0).all()
    plain = torch.empty((1, 90), device="cuda")
    nova.fourbit_mass(cache, q, lse, plain, ws, 90)
    assert torch.equal(plain[0, :70], m[0, :70])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 20, 140])
def test_queries_in_place(nova, dtype, n):
    """Queries as they lie in a joint projection's output, and with the heads in front of the rows."""
    g = torch.Generator().manual_seed(4)
    joint = torch.randn((2, n, 3 * 4, 64), generator=g).to(DTYPES[dtype]).cuda()
    a = _check_attention(nova, dtype, 2, 4, 2, 64, n, 150, 150, q=joint[:, :, :4])
    b = _check_attention(nova, dtype, 2, 4, 2, 64, n, 150, 150, q=joint[:, :, :4].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n", [1, 12, 140])
@pytest.mark.parametrize("scale", [0.0, -0.7, 6.0])
def test_wide_scores_and_other_scales(nova, dtype, dh, n, scale):
    """Scores of hundreds: the reference of the softmax moves from tile to tile; equal scores; a negative scale."""
    _check_attention(nova, dtype, 1, 2, 2, dh, n, 900, 900, scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n", [1, 140])
def test_rising_scores(nova, dtype, dh, n):
    """Every key outweighs all before it by far, then the other way round."""
    L = 500
    q = torch.zeros((1, n, 1, dh), dtype=DTYPES[dtype], device="cuda")
    q[..., 0] = 1.0
    for flip in (False, True):
        cache = FourBitCache.empty(1, 1, L, dh)
        k = torch.zeros((1, L, 1, dh), device="cuda")
        k[0, :, 0, 0] = torch.linspace(-400.0, 400.0, L, device="cuda")
        if flip:
            k = k.flip(1).contiguous()
        v = torch.randn((1, L, 1, dh), generator=torch.Generator().manual_seed(3)).cuda()
        nova.fourbit_append(cache, k, v, 0)
        out, lse = _run_attention(nova, cache, q, L, scale=1.0)
        K, V = (F.values(a.cpu().numpy(), s.cpu().numpy()) for a, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)))
        ref = F.attention(_np(q), K, V, 1.0, [L], [n])
        t_out, t_lse, _ = _bounds(ref, dtype, dh, L)
        assert (np.abs(_np(out) - ref[0]) <= t_out).all() and (np.abs(_np(lse) - ref[1]) <= t_lse).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 5, 150])
def test_nan_goes_where_it_belongs(nova, dtype, n):
    """A query of NaN spoils its own row; a cached row of NaN every query of its image and head, and no other."""
    B, H, hk, dh, L = 2, 4, 2, 64, 200
    cache, _ = _fill(B, hk, L, dh, [L] * B, 6)
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(7)).to(DTYPES[dtype]).cuda()
    q[0, n - 1, 1, 3] = float("nan")
    out, lse = _run_attention(nova, cache, q, L)
    bad = torch.isnan(out).all(-1)
    want = torch.zeros((B, n, H), dtype=torch.bool, device="cuda")
    want[0, n - 1, 1] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(out).any(-1), want) and torch.equal(torch.isnan(lse), want)
    q[0, n - 1, 1, 3] = 0.5
    cache.k_scales[1, 0, 130, 1] = 255
    out, lse = _run_attention(nova, cache, q, L)
    want[:] = False
    want[1, :, :2] = True
    assert torch.equal(torch.isnan(out).any(-1), want) and torch.equal(torch.isnan(lse), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 150])
def test_scores_of_minus_infinity_weigh_nothing(nova, dtype, n):
    """Keys whose score passes the end of fp32 from below, in front of and behind the finite ones."""
    L, dh = 600, 64
    q = torch.zeros((1, n, 1, dh), dtype=DTYPES[dtype], device="cuda")
    q[..., 0] = 100.0
    k = torch.zeros((1, L, 1, dh), device="cuda")
    k[0, :, 0, 1] = 1.0
    k[0, :200, 0, 0] = -2.0e38
    k[0, 300:, 0, 0] = -2.0e38
    v = torch.randn((1, L, 1, dh), generator=torch.Generator().manual_seed(3)).cuda()
    cache = FourBitCache.empty(1, 1, L, dh)
    nova.fourbit_append(cache, k, v, 0)
    out, lse = _run_attention(nova, cache, q, L, scale=1.0)
    V = F.values(cache.v_codes.cpu().numpy(), cache.v_scales.cpu().numpy())[0, 0, 200:300]
    assert np.abs(_np(out)[0, :, 0] - V.mean(0)).max() <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * np.abs(V).max()
    assert np.abs(_np(lse) - np.log(100.0)).max() <= 1e-5


@pytest.mark.parametrize("n", [1, 140])
def test_images_far_into_a_large_cache(nova, n):
    """The last images' rows lie past 2^32 bytes: the same bits as from a cache that holds their rows alone."""
    B, hk, cap, dh, L = 40, 8, 1 << 18, 128, 300
    cache = FourBitCache.empty(B, hk, cap, dh)
    small, _ = _fill(2, hk, cap=L, dh=dh, lens=[L] * 2, seed=8)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(cache, name)[B - 2:, :, :L] = getattr(small, name)
    q = torch.randn((2, n, hk, dh), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    big_q = torch.zeros((B, n, hk, dh), dtype=torch.bfloat16, device="cuda")
    big_q[B - 2:] = q
    lens = _ints([0] * (B - 2) + [L] * 2)
    out, lse = _run_attention(nova, cache, big_q, L, lens)
    ref, rlse = _run_attention(nova, small, q, L)
    assert (out[:B - 2] == 0).all()
    assert (out[B - 2:].float() - ref.float()).abs().max() <= 2.0 ** -7 * ref.float().abs().max()
    assert (lse[B - 2:] - rlse).abs().max() <= 1e-5
    k = torch.empty((B, 5, hk, dh), dtype=torch.bfloat16, device="cuda")
    nova.fourbit_unpack(cache, L - 5, k, None)
    sk = torch.empty((2, 5, hk, dh), dtype=torch.bfloat16, device="cuda")
    nova.fourbit_unpack(small, L - 5, sk, None)
    assert torch.equal(k[B - 2:], sk)
    nova.fourbit_append(cache, sk.expand(2, 5, hk, dh).repeat(B // 2, 1, 1, 1), k, cap - 5)
    nova.fourbit_unpack(cache, cap - 5, k, None)
    assert torch.equal(k[B - 2:], sk)


def test_one_image_with_a_very_long_cache(nova):
    """Two million rows, one query: many runs of keys, rows of one head past 2^27 bytes."""
    L, dh = 1 << 21, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = FourBitCache.empty(1, 1, L, dh)
    for r in range(0, L, 1 << 18):
        x = torch.randn((1, 1 << 18, 1, dh), generator=g, device="cuda")
        nova.fourbit_append(cache, x, x, r)
    q = torch.randn((1, 1, 2, dh), generator=g, device="cuda")
    out, lse = _run_attention(nova, cache, q, L)
    K = torch.empty((1, L, 1, dh), device="cuda")
    nova.fourbit_unpack(cache, 0, K, None)
    K = K[0, :, 0].double()
    s = (q[0, 0].double() @ K.T.contiguous()) * dh ** -0.5
    ref = torch.softmax(s, 1) @ K
    assert (lse[0, 0].double() - torch.logsumexp(s, 1)).abs().max() <= 2e-5
    assert (out[0, 0].double() - ref).abs().max() <= 2e-5 * (torch.softmax(s, 1) @ K.abs()).max()
    mass = torch.empty((1, L), device="cuda")
    ws = torch.empty(max(nova.fourbit_mass_workspace_bytes(cache, 2, 1, L), 16), dtype=torch.uint8, device="cuda")
    nova.fourbit_mass(cache, q, lse, mass, ws, L)
    p = torch.softmax(s, 1).sum(0)
    assert ((mass[0].double() - p).abs() <= 1e-4 * p).all()


# ---- eviction -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,hk,cap,cap2,kv_len,k", [(1, 1, 1, 1, 1, 1), (3, 5, 90, 40, 77, 33), (2, 2, 700, 700, 650, 600),
                                                   (2, 1, 50, 60, 50, 0)])
def test_evict(nova, dh, B, hk, cap, cap2, kv_len, k):
    print(f"fourbit evict dh={dh} B={B} hk={hk} {cap}->{cap2} kv_len={kv_len} k={k}", flush=True)
    g = np.random.default_rng(2)
    idx = np.stack([np.sort(g.permutation(kv_len)[:k]) for _ in range(B)]).astype(np.int32).reshape(B, k)
    if k > 2:
        idx[0, 1], idx[0, 2] = -1, kv_len                       # no rows of the image: zeros
    lens = [kv_len if b == 0 else kv_len // 2 for b in range(B)]
    counts = [k if b < 2 else k // 2 for b in range(B)]
    for lv, cv in ((None, None), (lens, counts)):
        lr, cr = lv or [kv_len] * B, cv or [k] * B
        src, hs = _fill(B, hk, cap, dh, [kv_len] * B, 5)
        dst, hd = _fill(B, hk, cap2, dh, [cap2] * B, 6)
        m_src = torch.rand((B, cap), generator=torch.Generator().manual_seed(1)).cuda()
        m_dst = torch.full((B, cap2), float("nan"), device="cuda")
        nxt = torch.full((B,), -7, dtype=torch.int32, device="cuda")
        nova.fourbit_evict(src, dst, torch.from_numpy(idx).cuda(), kv_len, k_per_row=None if cv is None else _ints(cv),
                           kv_len_per_row=None if lv is None else _ints(lv), kv_len_next=nxt, mass_src=m_src, mass_dst=m_dst)
        m = [min(a, c) for a, c in zip(lr, cr)]
        assert nxt.tolist() == m
        for half, old, got in ((hs[0], hd[0], (dst.k_codes, dst.k_scales)), (hs[1], hd[1], (dst.v_codes, dst.v_scales))):
            want = F.evict(half, old, idx, cr, lr)
            assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1])
        want_m = np.full((B, cap2), -1.0, dtype=np.float32)
        for b in range(B):
            for s in range(m[b]):
                want_m[b, s] = m_src[b, idx[b, s]].item() if 0 <= idx[b, s] < lr[b] else 0.0
        assert np.array_equal(m_dst.cpu().numpy(), want_m)


# ---- together -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attend_collect_select_evict_attend(nova, dtype):
    """A serving loop: append, attend, collect, keep the heaviest rows and the newest, go on with them."""
    B, H, hk, dh, cap, keep = 3, 4, 2, 64, 96, 40
    g = torch.Generator().manual_seed(21)
    lens = _ints([64, 50, 30])
    cache, halves = _fill(B, hk, cap, dh, [64, 50, 30], 13)
    K = [F.values(*halves[0])[b, :, :n] for b, n in enumerate((64, 50, 30))]
    V = [F.values(*halves[1])[b, :, :n] for b, n in enumerate((64, 50, 30))]
    mass = torch.full((B, cap), -1.0, device="cuda")
    heavy = [np.zeros(n) for n in (64, 50, 30)]
    for step in range(3):
        x = torch.randn((3, B, 1, max(H, hk), dh), generator=g).to(DTYPES[dtype]).cuda()
        k, v, q = x[0][:, :, :hk], x[1][:, :, :hk], x[2]
        after = torch.empty_like(lens)
        nova.fourbit_append(cache, k, v, 70, kv_len_per_row=lens, kv_len_next=after)
        lens = after
        for b in range(B):
            K[b] = np.concatenate([K[b], F.values(*F.quantise(_np(k)[b].transpose(1, 0, 2)))], 1)
            V[b] = np.concatenate([V[b], F.values(*F.quantise(_np(v)[b].transpose(1, 0, 2)))], 1)
            heavy[b] = np.append(heavy[b], 0.0)
        out, lse = _run_attention(nova, cache, q, 71, lens)
        ws = torch.empty(max(nova.fourbit_mass_workspace_bytes(cache, H, 1, 71), 16), dtype=torch.uint8, device="cuda")
        nova.fourbit_mass(cache, q, lse, mass, ws, 71, mass_in=mass, kv_len_per_row=lens)
        for b in range(B):
            n = K[b].shape[1]
            ref = F.attention(_np(q)[b:b + 1], K[b][None], V[b][None], dh ** -0.5, [n], [1])
            t_out, t_lse, d = _bounds(ref, dtype, dh, n)
            assert (np.abs(_np(out)[b:b + 1] - ref[0]) <= t_out).all()
            heavy[b] += F.mass(_np(q)[b:b + 1], K[b][None], dh ** -0.5, ref[1], None, [n], [1])[1][0]
            assert (np.abs(_np(mass)[b, :n] - heavy[b]) <= 1e-4 * heavy[b] + 1e-7).all()
    # the newest row stays whatever it has collected
    for b in range(B):
        mass[b, int(lens[b]) - 1] = float("inf")
    idx = torch.empty((B, keep), dtype=torch.int32, device="cuda")
    mask = torch.empty((B, cap), dtype=torch.uint8, device="cuda")
    nova.select(mass, keep, idx, mask)
    small = FourBitCache.empty(B, hk, 48, dh)
    m_small = torch.empty((B, 48), device="cuda")
    after = torch.empty_like(lens)
    nova.fourbit_evict(cache, small, idx, 73, kv_len_per_row=lens, kv_len_next=after, mass_src=mass, mass_dst=m_small)
    assert after.tolist() == [min(keep, n) for n in lens.tolist()]
    q = torch.randn((B, 1, H, dh), generator=g).to(DTYPES[dtype]).cuda()
    out, lse = _run_attention(nova, small, q, keep, after)
    for b in range(B):
        rows = idx[b, :int(after[b])].cpu().numpy()
        assert rows[-1] == int(lens[b]) - 1 and np.isinf(_np(m_small)[b, int(after[b]) - 1])
        ref = F.attention(_np(q)[b:b + 1], K[b][None][:, :, rows], V[b][None][:, :, rows], dh ** -0.5, [len(rows)], [1])
        t_out, t_lse, _ = _bounds(ref, dtype, dh, keep)
        assert (np.abs(_np(out)[b:b + 1] - ref[0]) <= t_out).all() and (np.abs(_np(lse)[b:b + 1] - ref[1]) <= t_lse).all()


@pytest.mark.parametrize("n,L", [(1, 1500), (1, 90), (40, 600), (300, 300)])
def test_captured_and_replayed(nova, n, L):
    """append, attention, mass and evict in one graph, replayed between eager calls on a workspace of their own: the same bits
    every time; and the same bits on another stream."""
    B, H, hk, dh = 2, 4, 2, 128
    cache, _ = _fill(B, hk, L + 8, dh, [L] * B, 3)
    g = torch.Generator().manual_seed(5)
    q = torch.randn((B, n, H, dh), generator=g).to(torch.bfloat16).cuda()
    new = torch.randn((B, 8, hk, dh), generator=g).to(torch.bfloat16).cuda()
    idx = torch.arange(0, L, 2, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    lens = _ints([L, L - 40])
    nws = max(nova.fourbit_attention_workspace_bytes(cache, H, n, L + 8), nova.fourbit_mass_workspace_bytes(cache, H, n, L + 8), 16)

    def buffers():
        return {"out": torch.empty((B, n, H, dh), dtype=torch.bfloat16, device="cuda"), "lse": torch.empty((B, n, H), device="cuda"),
                "mass": torch.empty((B, L + 8), device="cuda"), "dst": FourBitCache.empty(B, hk, idx.shape[1], dh),
                "len": torch.empty(B, dtype=torch.int32, device="cuda"), "len2": torch.empty(B, dtype=torch.int32, device="cuda"),
                "ws": torch.full((nws,), 255, dtype=torch.uint8, device="cuda")}

    def go(b):
        nova.fourbit_append(cache, new, new, L, kv_len_per_row=lens, kv_len_next=b["len"])
        nova.fourbit_attention(cache, q, b["out"], b["ws"], L + 8, lse=b["lse"], kv_len_per_row=b["len"])
        nova.fourbit_mass(cache, q, b["lse"], b["mass"], b["ws"], L + 8, kv_len_per_row=b["len"])
        nova.fourbit_evict(cache, b["dst"], idx, L + 8, kv_len_per_row=b["len"], kv_len_next=b["len2"])

    def results(b):
        return [b[k].clone() for k in ("out", "lse", "mass", "len", "len2")] + [b["dst"].k_codes.clone(), b["dst"].v_scales.clone()]

    eager, held = buffers(), buffers()
    go(eager)
    torch.cuda.synchronize()
    want = results(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(held)
    for _ in range(4):
        for t in (held["out"], held["lse"], held["mass"]):
            t.fill_(float("nan"))
        graph.replay()
        go(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(held), want))
        assert all(torch.equal(a, b) for a, b in zip(results(eager), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(held)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(results(held), want))


def test_two_streams_at_once(nova):
    """Two calls that overlap, each with buffers of its own."""
    args = []
    for i, (n, L) in enumerate(((1, 4000), (200, 900))):
        cache, _ = _fill(2, 2, L, 64, [L] * 2, i)
        q = torch.randn((2, n, 4, 64), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda()
        args.append((cache, q, L, torch.empty_like(q),
                     torch.empty(max(nova.fourbit_attention_workspace_bytes(cache, 4, n, L), 16), dtype=torch.uint8, device="cuda")))
    want = [_run_attention(nova, c, q, L)[0] for c, q, L, _, _ in args]
    streams = [torch.cuda.Stream() for _ in args]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (c, q, L, out, ws) in zip(streams, args):
            with torch.cuda.stream(s):
                nova.fourbit_attention(c, q, out, ws, L)
    torch.cuda.synchronize()
    assert all(torch.equal(a[3], w) for a, w in zip(args, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,L", [(8, 40), (40, 300), (300, 2300)])
def test_padding_behind_the_live_queries_is_nobodys(nova, dtype, n, L):
    """NaN and infinities in the padded slots of a batch: the live queries get the bits they get with zeros there, and the weights
    collected are the same."""
    B, H, hk, dh = 3, 4, 2, 64
    cache, _ = _fill(B, hk, L, dh, [L] * B, 6)
    counts = _ints([n, n // 2, 1])
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(7)).to(DTYPES[dtype]).cuda()
    got = []
    for pad in (0.0, float("nan"), float("inf")):
        for b, c in enumerate(counts.tolist()):
            q[b, c:] = pad
        out, lse = _run_attention(nova, cache, q, L, counts=counts)
        mass = torch.empty((B, L), device="cuda")
        ws = torch.empty(max(nova.fourbit_mass_workspace_bytes(cache, H, n, L), 16), dtype=torch.uint8, device="cuda")
        nova.fourbit_mass(cache, q, lse, mass, ws, L, n_per_row=counts)
        got.append((out, lse, mass))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spoil", ["query", "key"])
@pytest.mark.parametrize("n", [1, 12, 40, 600])
def test_weights_that_are_no_numbers_leave_an_image_its_rows(nova, dtype, spoil, n):
    """A query or a key of NaN makes every weight of its image NaN: its rows keep what they had collected, in front of the rows
    that it does not have, and eviction finds them.  The other image gets the bits it gets without."""
    B, H, hk, dh, cap, keep = 2, 4, 2, 64, 90, 60
    lens = [50, 90]
    cache, halves = _fill(B, hk, cap, dh, lens, 17)
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(18)).to(DTYPES[dtype]).cuda()
    m_in = torch.rand((B, cap), generator=torch.Generator().manual_seed(19)).cuda()
    m_in[:, ::5] = -1.0
    m_in[:, 7], m_in[:, 11] = float("inf"), float("nan")

    def weights():
        out, lse = _run_attention(nova, cache, q, cap, _ints(lens))
        mass = torch.full((B, cap), float("nan"), device="cuda")
        ws = torch.full((max(nova.fourbit_mass_workspace_bytes(cache, H, n, cap), 16),), 255, dtype=torch.uint8, device="cuda")
        nova.fourbit_mass(cache, q, lse, mass, ws, cap, mass_in=m_in, kv_len_per_row=_ints(lens))
        return mass

    clean = weights()
    if spoil == "query":
        q[0, n // 2, 3, 5] = float("nan")
    else:
        cache.k_scales[0, :, 20, 1] = 255
        halves[0][1][0, :, 20, 1] = 255
    mass = weights()
    before = torch.where(m_in > 0, m_in, 0.0)
    assert torch.equal(mass[0, :50], before[0, :50])          # a row's sum is over all key heads: NaN in one is NaN in all
    assert (mass[0, 50:] == -1).all() and torch.equal(mass[1], clean[1])
    idx = torch.empty((B, keep), dtype=torch.int32, device="cuda")
    mask = torch.empty((B, cap), dtype=torch.uint8, device="cuda")
    nova.select(mass, keep, idx, mask)
    dst = FourBitCache.empty(B, hk, keep, dh)
    m_dst = torch.empty((B, keep), device="cuda")
    after = torch.empty(B, dtype=torch.int32, device="cuda")
    nova.fourbit_evict(cache, dst, idx, cap, kv_len_per_row=_ints(lens), kv_len_next=after, mass_src=mass, mass_dst=m_dst)
    assert after.tolist() == [50, 60] and idx[0, :50].tolist() == list(range(50))
    assert torch.equal(m_dst[0, :50], mass[0, :50]) and (m_dst[0, 50:] == -1).all()
    for half, got in ((halves[0], (dst.k_codes, dst.k_scales)), (halves[1], (dst.v_codes, dst.v_scales))):
        assert all(np.array_equal(g[0, :, :50].cpu().numpy(), w[0, :, :50]) for g, w in zip(got, half))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n", [1, 20, 140])
def test_a_scale_of_zero_and_scores_without_bound(nova, dtype, dh, n):
    """Every row weighs the same, however large the finite scores are (around 2^115 here)."""
    q = 2.0 ** 112 * torch.randn((1, n, 2, dh), generator=torch.Generator().manual_seed(23))
    _check_attention(nova, dtype, 1, 2, 2, dh, n, 301, 300, scale=0.0, q=q.to(DTYPES[dtype]).cuda())


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n", [1, 20, 140])
def test_queries_at_the_end_of_fp32(nova, dh, n):
    """fp32 queries between the largest bf16 number and the largest fp32 one, scores of order one."""
    L = 130
    q = torch.zeros((1, n, 2, dh), device="cuda")
    q[..., 3], q[..., dh - 1] = torch.finfo(torch.float32).max, -3.397e38
    cache = FourBitCache.empty(1, 2, L, dh)
    g = torch.Generator().manual_seed(29)
    k, v = (torch.randn((1, L, 2, dh), generator=g).cuda() for _ in range(2))
    k = k.clamp(-1, 1) * 0.25
    nova.fourbit_append(cache, k, v, 0)
    scale = 2.0 ** -126
    out, lse = _run_attention(nova, cache, q, L, scale=scale)
    K, V = (F.values(a.cpu().numpy(), s.cpu().numpy()) for a, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)))
    ref = F.attention(_np(q), K, V, scale, [L], [n])
    t_out, t_lse, d = _bounds(ref, "f32", dh, L)
    assert (np.abs(_np(out) - ref[0]) <= t_out).all() and (np.abs(_np(lse) - ref[1]) <= t_lse).all()
    mass = torch.empty((1, L), device="cuda")
    ws = torch.empty(max(nova.fourbit_mass_workspace_bytes(cache, 2, n, L), 16), dtype=torch.uint8, device="cuda")
    nova.fourbit_mass(cache, q, lse, mass, ws, L, scale=scale)
    want, got = F.mass(_np(q), K, scale, _np(lse), None, [L], [n])
    assert (np.abs(_np(mass) - want) <= got * (2 * d.max() + (2 * n + 128) * U) + 2 * U * want).all()


def _check_weights(nova, dtype, B, H, hk, dh, n, L, lens=None, counts=None, seed=31):
    """The weights alone, of any logarithms, at a closer bound: a sum is a chain of 32 numbers of a tile, one addition per tile of a
    run (33 here) and one of the lane's halves, of an eighth of the parts (66), of eight groups and of what was there: fewer than
    256 roundings of numbers that are none of them negative."""
    print(f"fourbit weights {dtype} B={B} H={H}/{hk} dh={dh} n={n} L={L} lens={lens} counts={counts}", flush=True)
    real, live = lens or [L] * B, counts or [n] * B
    cache, halves = _fill_codes(B, hk, L + 1, dh, real, seed)
    g = torch.Generator().manual_seed(seed)
    q = (0.05 * torch.randn((B, n, H, dh), generator=g)).to(DTYPES[dtype]).cuda()
    lse = (np.log(L) + torch.randn((B, n, H), generator=g)).cuda()
    m_in = torch.rand((B, L + 1), generator=g).cuda()
    ws = torch.full((max(nova.fourbit_mass_workspace_bytes(cache, H, n, L), 16),), 255, dtype=torch.uint8, device="cuda")
    mass = torch.full((B, L + 1), float("nan"), device="cuda")
    nova.fourbit_mass(cache, q, lse, mass, ws, L, mass_in=m_in, n_per_row=None if counts is None else _ints(counts),
                      kv_len_per_row=None if lens is None else _ints(lens))
    q64, K, sc = _np(q), _values(halves[0], real), dh ** -0.5
    want, got = F.mass(q64, K, sc, _np(lse), _np(m_in), real, live)
    reach = max(sc * (np.abs(q64[b, :live[b], h]) @ np.abs(K[b, h // (H // hk), :real[b]]).T).max(initial=0)
                for b in range(B) for h in range(H))
    d = (2 * dh + 32) * U * (reach + float(lse.abs().max()) + 1)
    diff = np.abs(_np(mass) - want)
    assert (diff <= got * (2 * d + 256 * U) + 2 * U * np.abs(want)).all(), (diff / np.maximum(got, 1e-30)).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,H,hk,n,L", [(3, 90, 90, 521, 3), (2, 390, 130, 187, 5), (1, 2080, 260, 70, 257), (2, 300, 150, 531, 40)])
def test_weights_of_runs_with_many_tiles(nova, dtype, dh, B, H, hk, n, L):
    """More chunks of keys than CUs: all tiles of rows in one run, or in two with a shorter second; one, two, three and eight heads
    to a key head, so that the walk over rows wraps inside tiles and between them; images with fewer rows and keys."""
    _check_weights(nova, dtype, B, H, hk, dh, n, L)
    if B > 1:
        _check_weights(nova, dtype, B, H, hk, dh, n, L, lens=[L, L // 2, 1][:B], counts=[n - 1, n, n // 3][:B])


@pytest.mark.parametrize("dtype,dh,H,hk,L", [("bf16", 64, 60, 30, 2500), ("bf16", 128, 30, 15, 5000), ("f32", 64, 60, 30, 2500)])
def test_weights_of_several_runs_with_many_tiles(nova, dtype, dh, H, hk, L):
    """Four runs of nine tiles of 64 rows (of 17 of 32 in fp32), the last one shorter."""
    _check_weights(nova, dtype, 1, H, hk, dh, 1050, L)
