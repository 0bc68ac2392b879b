"""GPU parity of the pruned block whose cache is held in 4 bits, and of the image runner on such caches.

The block's own rows are quantised on the device, so the float64 block is given the cached rows as they read afterwards; that the
rows are those of the block's keys and values is checked apart: within half a step of the 4-bit levels (largest gap 2 of a
largest magnitude of at least 3, the scale being the smallest that reaches: 1 / 3 of the group's largest magnitude), on top of
the tolerance of the projection.  Tolerances of the block itself as everywhere: max|d| / max|ref| of 2e-2 (bf16) and 2e-5 (fp32)."""
import numpy as np
import pytest
import torch

import workloads as WL
from oracle import nova_fourbit as F
from paper_2602_01345_amd import BlockShape, BlockVariant, FourBitCache, NOVA_BF16, NOVA_F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hx():
    import harness
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU and the built libnova.so (no fallback)")
    return harness


def _ints(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device="cuda")


def _cross(hx, hb, heads):
    """Device side of a cross-attention sub-layer; what lies behind the condition tokens is NaN."""
    c = hb.variant["cross"]
    n = c["k_text"].shape[1]
    cap = (n + 63) // 64 * 64
    return {"text_len": n, "k_text": hx.pack_k_cache(c["k_text"].cuda(), heads, cap, float("nan")),
            "v_text": hx.pack_v_cache(c["v_text"].cuda(), heads, cap, float("nan")),
            **{w: c[w].cuda() for w in ("w_cq", "b_cq", "w_co", "b_co")}}


def _check(hx, dtype, C, heads, B, grid, P, k, counts=None, lens=None, variant=None, cap_extra=3, seed=31):
    print(f"fourbit block {dtype} C={C} heads={heads} B={B} P={P} k={k} counts={counts} lens={lens} {variant}", flush=True)
    wl = WL.Workload("fourbit", dtype, B=B, C=C, heads=heads, L=1, V=64, keep_hi=.5, keep_lo=.5,
                     scales=(WL.Scale(grid=grid, prev_grid=grid - 1, kv_len=P),), seed=seed)
    hb = hx.make_host_block(wl, 0, k=k, variant=variant)
    nova, tdt, dh = hx.nova(), WL.torch_dtype(dtype), C // heads
    cap = P + k + cap_extra
    real, live = lens or [P] * B, counts or [k] * B
    cache = FourBitCache.empty(B, heads, cap, dh)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(cache, name).fill_(255)
    rows = lambda t: t.cuda().reshape(B, P, heads, dh)
    if P:
        nova.fourbit_append(cache, rows(hb.k_prior), rows(hb.v_prior), 0, n_per_row=_ints(real))
    before = {n: getattr(cache, n).clone() for n in ("k_codes", "k_scales", "v_codes", "v_scales")}
    idx = np.stack([np.sort(np.random.default_rng(b).permutation(grid * grid)[:k]) for b in range(B)]).astype(np.int32)
    idx = idx.reshape(B, k)
    for b in range(B):
        idx[b, live[b]:] = -1
    var = None
    if hb.variant:
        qs, ada = hb.variant.get("qk_scale"), hb.variant.get("ada")
        var = BlockVariant(gelu_tanh=bool(hb.variant.get("gelu_tanh", False)), qk_scale=None if qs is None else qs.cuda(),
                           ada=None if ada is None else ada.cuda())
        if hb.variant.get("cross") is not None:
            var.cross = _cross(hx, hb, heads)
    shape = BlockShape(NOVA_BF16 if dtype == "bf16" else NOVA_F32, B, grid * grid, C, heads, P, cap, k)
    ws = torch.full((nova.fourbit_block_workspace_bytes(shape),), 255, dtype=torch.uint8, device="cuda")
    y = torch.full((B, k, C), float("nan"), dtype=tdt, device="cuda")
    mass = torch.full((B, cap), float("nan"), device="cuda")
    m_in = torch.rand((B, cap), generator=torch.Generator().manual_seed(2)).cuda()
    nxt = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    W = {n: t.cuda() for n, t in hb.weights.items()}
    nova.pruned_block_fourbit(shape, W, var, None if counts is None else _ints(counts), None if lens is None else _ints(lens), nxt,
                              hb.x.cuda(), torch.from_numpy(idx).cuda(), cache, y, ws, mass, m_in)
    torch.cuda.synchronize()
    assert nxt.tolist() == [a + c for a, c in zip(real, live)]
    total = [a + c for a, c in zip(real, live)]
    K, V = (F.values(a.cpu().numpy(), s.cpu().numpy()) for a, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)))
    kw = {}
    if hb.variant:
        kw = dict(gelu_form="tanh" if hb.variant.get("gelu_tanh") else "erf",
                  qk_scale=None if hb.variant.get("qk_scale") is None else hx.f64(hb.variant["qk_scale"]),
                  ada=None if hb.variant.get("ada") is None else hx.f64(hb.variant["ada"]))
        if hb.variant.get("cross") is not None:
            kw["cross"] = {n: hx.f64(t) for n, t in hb.variant["cross"].items()}
    ry, rk, rv, got = F.block(hx.f64(hb.x), idx, {n: hx.f64(t) for n, t in hb.weights.items()}, K, V, heads, total, live, **kw)
    tol = hx.BF16_TOL if dtype == "bf16" else hx.F32_TOL
    err = max(float(np.abs(hx.f64(y[b, :live[b]]) - ry[b, :live[b]]).max()) for b in range(B) if live[b])
    assert err <= tol * np.abs(ry).max(), err
    for half, ref in ((K, rk), (V, rv)):
        for b in range(B):
            new = half[b, :, real[b]:total[b]].transpose(1, 0, 2).reshape(live[b], C)
            grp = np.abs(ref[b, :live[b]]).reshape(live[b], C // 32, 32).max(-1, initial=0).repeat(32, -1)
            assert (np.abs(new - ref[b, :live[b]]) <= grp / 3 + tol * np.abs(ref).max()).all()
    for n, t in before.items():                               # nothing but the images' own new rows is written
        now = getattr(cache, n)
        for b in range(B):
            assert torch.equal(now[b, :, :real[b]], t[b, :, :real[b]]) and torch.equal(now[b, :, total[b]:], t[b, :, total[b]:])
    m = hx.f64(mass)
    for b in range(B):
        want = hx.f64(m_in)[b, :total[b]] + got[b, :total[b]]
        assert np.abs(m[b, :total[b]] - want).max(initial=0) <= tol * max(want.max(initial=0), 1.0)
        assert (m[b, total[b]:] == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,heads", [(128, 2), (256, 2)])
@pytest.mark.parametrize("B,grid,P,k", [(1, 5, 0, 25), (2, 9, 33, 40), (2, 17, 300, 200), (2, 6, 150, 1)])
def test_block(hx, dtype, C, heads, B, grid, P, k):
    _check(hx, dtype, C, heads, B, grid, P, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("variant", [{"qk_norm"}, {"gelu_tanh", "ada"}, {"qk_norm", "gelu_tanh", "ada"}])
def test_variants(hx, dtype, variant):
    _check(hx, dtype, 128, 2, 2, 9, 0, 50, variant=variant)
    if "qk_norm" not in variant:
        _check(hx, dtype, 128, 2, 2, 9, 70, 50, variant=variant)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P,k", [(90, 60), (300, 200)])
def test_images_with_their_own_counts(hx, dtype, P, k):
    _check(hx, dtype, 128, 2, 4, 15, P, k, counts=[k, 0, 7, k // 2], lens=[P, 5, 0, P // 3])


def test_a_block_without_kept_tokens_does_nothing(hx):
    nova = hx.nova()
    cache = FourBitCache.empty(1, 2, 10, 64)
    shape = BlockShape(NOVA_BF16, 1, 4, 128, 2, 5, 10, 0)
    assert nova.fourbit_block_workspace_bytes(shape) == 0
    t = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    W = {n: t for n in ("w_qkv", "w_o", "w_fc1", "w_fc2")}
    nova.pruned_block_fourbit(shape, W, None, None, None, None, t, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), cache, t,
                              torch.empty(256, dtype=torch.uint8, device="cuda"))


# ---- the runner -----------------------------------------------------------------------------------------------------
GRIDS = [1, 2, 3, 5, 7]


def _runner(hx, dtype, evict_to, B=2, L=3, C=128, heads=2):
    from paper_2602_01345_amd.image import ImageRunner
    scales = tuple(WL.Scale(grid=g, prev_grid=GRIDS[max(t - 1, 0)], kv_len=sum(q * q for q in GRIDS[:t])) for t, g in enumerate(GRIDS))
    wl = WL.Workload("fourbit-chain", dtype, B=B, C=C, heads=heads, L=L, V=64, keep_hi=.7, keep_lo=.4, scales=scales, seed=5)
    W = [{n: t.cuda() for n, t in WL.make_weights(wl, j).items()} for j in range(L)]
    r = ImageRunner(hx.nova(), B=B, C=C, heads=heads, grids=GRIDS, dtype=WL.torch_dtype(dtype), weights=W, cache_bits=4,
                    evict_to=evict_to)
    xs = [WL.make_x(wl, s).cuda() for s in scales]
    logits = [[WL.make_logits(wl, j, s).cuda() for j in range(L)] for s in scales]
    tables = {t: [WL.keep_count(wl.keep_ratio(j), GRIDS[t] ** 2) for j in range(L)] for t in (3, 4)}
    return r, xs, logits, tables


def _run(r, xs, logits, tables):
    return [r.run_scale(t, xs[t], logits=logits[t], k_table=tables.get(t), keep_cache=t >= 2) for t in range(len(GRIDS))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("evict_to", [None, 12])
def test_runner_is_its_calls_one_by_one(hx, dtype, evict_to):
    """All scales of an image, and of a second one after reset(), against the same calls written out on caches that are never
    swapped: the same bits."""
    r, xs, logits, tables = _runner(hx, dtype, evict_to)
    n, B, L, C, heads = r.nova, r.B, r.L, r.C, r.heads
    for _ in range(2):
        r.reset()
        results = _run(r, xs, logits, tables)
        caches = [FourBitCache.empty(B, heads, sum(g * g for g in GRIDS), C // heads) for _ in range(L)]
        mass = [torch.full((B, c.capacity), -1.0, device="cuda") for c in caches]
        have = [0] * L
        for t, g in enumerate(GRIDS):
            N, x = g * g, xs[t]
            for j in range(L):
                k = tables[t][j] if t in tables else N
                idx = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
                mask = torch.ones((B, N), dtype=torch.uint8, device="cuda")
                if t in tables:
                    H = torch.empty((B, N), device="cuda")
                    idx = torch.empty((B, k), dtype=torch.int32, device="cuda")
                    n.entropy(logits[t][j], H)
                    n.select(H, k, idx, mask)
                shape = BlockShape(r.code, B, N, C, heads, have[j], caches[j].capacity, k)
                y = torch.empty((B, k, C), dtype=x.dtype, device="cuda")
                ws = torch.empty(n.fourbit_block_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
                n.pruned_block_fourbit(shape, r.weights[j], None, None, None, None, x, idx, caches[j], y, ws, mass[j], mass[j])
                have[j] += k
                out = torch.empty_like(x)
                prev = results[t - 1].block_cache[j] if t else None
                pg = GRIDS[t - 1] if t and prev is not None else g
                n.merge_cache(g, g, pg, pg, k, x, y, idx, mask, prev, out)
                assert torch.equal(out, results[t].block_out[j]), (t, j)
                x = out
            for j in range(L):
                if evict_to is not None and have[j] > evict_to and t + 1 < len(GRIDS):
                    kept = torch.empty((B, evict_to), dtype=torch.int32, device="cuda")
                    m8 = torch.empty(mass[j].shape, dtype=torch.uint8, device="cuda")
                    n.select(mass[j], evict_to, kept, m8)
                    dst, dm = FourBitCache.empty(B, heads, caches[j].capacity, C // heads), torch.empty_like(mass[j])
                    n.fourbit_evict(caches[j], dst, kept, have[j], mass_src=mass[j], mass_dst=dm)
                    caches[j], mass[j], have[j] = dst, dm, evict_to
        assert r.kv_len == have and all(rows.tolist() == [h] * B for rows, h in zip(r.kv_rows, have))
    if evict_to is not None:
        assert r.cap < sum(g * g for g in GRIDS)


@pytest.mark.parametrize("evict_to", [None, 12])
def test_planned_scales_and_their_graphs(hx, evict_to):
    """The planned form, eager and as one graph per scale replayed for several images, gives the bits of the eager runner."""
    r, xs, logits, tables = _runner(hx, "bf16", evict_to)
    want = [[s.out.clone() for s in (_run(r, x, logits, tables), r.reset())[0]] for x in (xs, [t.flip(1) for t in xs])]
    plans = r.plan_image(tables, {t: logits[t] for t in tables}, 2)
    for p in plans:
        p.x.copy_(xs[p.t])
    for captured in (False, True):
        if captured:
            for p in plans:
                r.capture(p)
        for i, images in enumerate((xs, [t.flip(1) for t in xs], xs)):
            for p, w in zip(plans, want[i % 2]):
                p.x.copy_(images[p.t])
                assert torch.equal(r.launch(p), w), (captured, i, p.t)


def test_counts_of_the_controller_with_eviction(hx):
    """Every image has its own keep counts and cache lengths; nothing reads a row that is not an image's own."""
    r, xs, logits, tables = _runner(hx, "bf16", 12)
    for st in r.stores + [r._spare]:
        for nme in ("k_codes", "k_scales", "v_codes", "v_scales"):
            getattr(st.cache, nme).fill_(255)                 # NaN wherever no row has been written
    ratio = torch.tensor([0.2, 0.8], device="cuda")
    for t in range(len(GRIDS)):
        res = r.run_scale(t, xs[t], logits=logits[t], ratio_t=ratio if t >= 3 else None, keep_cache=t >= 2)
        assert torch.isfinite(res.out.float()).all()
        if t >= 3:
            assert all(len(set(k.tolist())) == 2 for k in res.k)
    assert all(0 < n <= r.cap for rows in r.kv_rows for n in rows.tolist())


def test_an_image_of_nan_keeps_its_rows_and_leaves_the_other_alone(hx):
    """One image's tokens are NaN at a scale: eviction still takes rows that the image has, never one made of zeros, and the other
    image gets the bits that it gets without."""
    got = []
    for spoil in (False, True):
        r, xs, logits, tables = _runner(hx, "bf16", 12)
        for st in r.stores + [r._spare]:
            for nme in ("k_codes", "k_scales", "v_codes", "v_scales"):
                getattr(st.cache, nme).fill_(0)               # scale byte 0: not the 127 of a row made of zeros
        ratio = torch.tensor([0.9, 0.2], device="cuda")
        outs = []
        for t in range(len(GRIDS)):
            x = xs[t].clone()
            if spoil and t == 3:
                x[0] = float("nan")
            outs.append(r.run_scale(t, x, logits=logits[t], ratio_t=ratio if t >= 3 else None, keep_cache=t >= 2).out[1])
            if t == 3:
                for st in r.stores:
                    for b, rows in enumerate(st.rows.tolist()):
                        made = (st.cache.k_codes[b, 0, :rows] == 0).all(-1) & (st.cache.k_scales[b, 0, :rows] == 127).all(-1)
                        assert rows == 12 and not made.any()
                        assert (st.mass[b, :rows] >= 0).all() and (st.mass[b, rows:] == -1).all()
        got.append(outs)
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("variant", [{"qk_norm"}, {"cross"}, {"cross", "gelu_tanh", "ada"}, {"qk_norm", "gelu_tanh", "ada", "cross"}])
@pytest.mark.parametrize("C,heads,P,k", [(128, 2, 70, 50), (256, 2, 600, 130)])
def test_variants_over_prior_rows(hx, dtype, variant, C, heads, P, k):
    """Unit-length keys in front of the block's own, cross-attention behind the attention over the 4-bit cache, all of it at once;
    then with images that have lengths and counts of their own."""
    _check(hx, dtype, C, heads, 2, 13, P, k, variant=variant)
    _check(hx, dtype, C, heads, 4, 13, P, k, counts=[k, 1, 0, k // 3], lens=[P, 0, 7, P // 2], variant=variant)


@pytest.mark.parametrize("evict_to", [None, 12, 4])
def test_scales_captured_in_the_middle_of_an_image(hx, evict_to):
    """Every scale is recorded when the image has come to it, then launched: recording leaves the caches, the weights and the row
    counts as they were.  The graphs then serve further images."""
    r, xs, logits, tables = _runner(hx, "bf16", evict_to)
    want = [s.out.clone() for s in _run(r, xs, logits, tables)]
    r.reset()
    plans = r.plan_image(tables, {t: logits[t] for t in tables}, 2)
    for image in range(3):
        for p, w in zip(plans, want):
            p.x.copy_(xs[p.t])
            if image == 0:
                r.capture(p)
            assert torch.equal(r.launch(p), w), (image, p.t)
