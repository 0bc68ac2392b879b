"""Operators on a key/value cache held in 4 bits: what is measured of them, and their plain forms.

The cache holds K and V of every (image, key head) as rows of `dh` channels: two 4-bit codes per byte (low nibble first;
code = sign, then one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one scale byte per 32 channels (2^(byte - 127), 255: NaN).

  append   quantises new rows behind the ones an image has, and reads them back as the values they stand for
  attend   attention of n queries per image over the cached rows, with the logarithm of each softmax sum; heads may share
           keys, images may have lengths of their own
  mass     attention weight that every cached row collects from n queries, summed over queries and heads, on top of what it
           had collected before
  evict    the rows in a list move to the front of another cache, with what they have collected, and are read back

Sizes are those of this repository's workloads (256- to 1024-pixel scale lists) and generic ones for serving token by token.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZES = {"f32": 4, "bf16": 2}
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_NOVA = None


# ---- the cases ------------------------------------------------------------------------------------------------------
def _append(name, dtype, B, kv_heads, dh, n, kv_len, source, ragged=False):
    return {"name": name, "kind": "append", "dtype": dtype, "B": B, "kv_heads": kv_heads, "dh": dh, "n": n,
            "kv_len": kv_len, "source": source, "ragged": ragged}


def _attend(name, dtype, B, heads, kv_heads, dh, n, kv_len, ragged=False, packed_q=False, kind="attend"):
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "heads": heads, "kv_heads": kv_heads, "dh": dh, "n": n,
            "kv_len": kv_len, "ragged": ragged, "packed_q": packed_q}


def _evict(name, B, kv_heads, dh, kv_len, k, ragged=False):
    return {"name": name, "kind": "evict", "dtype": "bf16", "B": B, "kv_heads": kv_heads, "dh": dh, "kv_len": kv_len, "k": k,
            "ragged": ragged}


def listed():
    return [
        # one new row per image of a batch, every image with a length of its own: the least there is to append
        _append("append-token-b8", "bf16", 8, 16, 64, 1, 679, "rows", ragged=True),
        # the whole prior cache of two 1024-pixel images, from the 16-bit cache layouts (values key-minor)
        _append("append-1024px-prior", "bf16", 2, 16, 128, 6425, 0, "caches"),
        # an odd number of fp32 rows as they lie in the output of a joint projection of queries, keys and values
        _append("append-f32-odd", "f32", 3, 5, 64, 333, 250, "joint"),
        # one query per image against the prior rows of a 256-pixel image: the smallest attention, latency
        _attend("attend-token-256px", "bf16", 8, 16, 16, 64, 1, 424),
        # token by token over long caches of different lengths, four query heads to a key head
        _attend("attend-token-32k", "bf16", 4, 32, 8, 128, 1, 32768, ragged=True),
        # a handful of fp32 queries against all rows before the scale 40 x 40
        _attend("attend-few-f32", "f32", 2, 16, 16, 64, 5, 2521, packed_q=True),
        # last scale of 512-pixel images, half of the tokens kept, images of different lengths, 36 heads
        _attend("attend-512px-b8", "bf16", 8, 36, 36, 64, 512, 1728, ragged=True),
        # last scale of two 1024-pixel images, the tokens kept by the first block: the largest
        _attend("attend-1024px-b2", "bf16", 2, 16, 16, 128, 2458, 8883),
        # what one token per image adds to the weights of long caches
        _attend("mass-token-32k", "bf16", 4, 32, 8, 128, 1, 32768, ragged=True, kind="mass"),
        # what the tokens kept by a middle block at the last scale of two 1024-pixel images add
        _attend("mass-1024px-b2", "bf16", 2, 16, 16, 128, 1640, 8065, kind="mass"),
        # half of the rows of eight 256-pixel images stay
        _evict("evict-256px-b8", 8, 16, 64, 680, 340),
        # a quarter of four long caches of different lengths stays
        _evict("evict-32k", 4, 8, 128, 32768, 8192, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def draw(rng):
    """One more case of the same ranges; never dearer than the largest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(("append", "attend", "attend", "attend", "mass", "mass", "evict"))
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        dh = rng.choice((64, 128))
        B = _log_int(rng, 1, 16)
        kv_heads = _log_int(rng, 1, 36)
        ragged = rng.random() < 0.5
        if kind == "append":
            case = {"kind": kind, "dtype": dtype, "B": B, "kv_heads": kv_heads, "dh": dh, "n": _log_int(rng, 1, 8192),
                    "kv_len": rng.randint(0, 4096), "source": rng.choice(("rows", "joint", "caches")), "ragged": ragged}
        elif kind == "evict":
            kv_len = _log_int(rng, 16, 32768)
            case = {"kind": kind, "dtype": "bf16", "B": B, "kv_heads": kv_heads, "dh": dh, "kv_len": kv_len,
                    "k": rng.randint(1, kv_len), "ragged": ragged}
        else:
            group = rng.choice((1, 1, 2, 3, 4, 8))
            n = 1 if rng.random() < 0.3 else _log_int(rng, 1, 4096)
            case = {"kind": kind, "dtype": dtype, "B": B, "heads": kv_heads * group, "kv_heads": kv_heads, "dh": dh, "n": n,
                    "kv_len": _log_int(rng, 1, 32768), "ragged": ragged, "packed_q": rng.random() < 0.3}
        if _cost(case) <= most:
            return case


def work(case):
    B, hk, dh = case["B"], case["kv_heads"], case["dh"]
    row = dh // 2 + dh // 32                                     # bytes of one cached row of K or of V
    e = _SIZES[case["dtype"]]
    if case["kind"] == "append":
        rows = 2 * B * case["n"] * hk                            # rows in; codes and scales out; values out
        return {"bytes": rows * (dh * e + row + dh * e), "flops": 0}
    lens = sum(_lengths(case))
    if case["kind"] == "evict":
        rows = 2 * sum(min(case["k"], n) for n in _lengths(case)) * hk
        return {"bytes": rows * (2 * row + dh * e) + lens * 4, "flops": 0}
    H, n = case["heads"], case["n"]
    if case["kind"] == "attend":
        return {"bytes": 2 * lens * hk * row + 2 * B * n * H * dh * e + B * n * H * 4, "flops": 4 * n * H * lens * dh}
    return {"bytes": lens * hk * row + B * n * H * (dh * e + 4) + 2 * lens * 4, "flops": 2 * n * H * lens * dh}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Rows every image has in the cache.  "ragged": from the full length down to a quarter of it, spread evenly."""
    B, L = case["B"], case["kv_len"]
    if not case["ragged"]:
        return [L] * B
    return [L - (3 * L * b) // (4 * B) for b in range(B)]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(g, shape):
    """fp32 rows [..., heads, dh], N(0, 1) with channels of different reach, as keys and values have them."""
    reach = torch.exp(0.5 * torch.randn(shape[-2:], generator=g, device="cuda"))
    return torch.randn(shape, generator=g, device="cuda") * reach


def _cache_inputs(case, g):
    """Codes and scales of the images' rows; whatever lies behind them is left as memory may hold it (all ones)."""
    B, hk, dh, L = case["B"], case["kv_heads"], case["dh"], case["kv_len"]
    lens = torch.tensor(_lengths(case), device="cuda")
    live = (torch.arange(L, device="cuda") < lens[:, None])[:, None, :, None]
    out = []
    for _ in range(2):
        codes, scales = _quantise(_rows(g, (B, L, hk, dh)).permute(0, 2, 1, 3))
        out += [torch.where(live, codes, 255).to(torch.uint8).contiguous(),
                torch.where(live, scales, 255).to(torch.uint8).contiguous()]
    return out


def _inputs(case, seed):
    g = _generator(seed)
    B, hk, dh = case["B"], case["kv_heads"], case["dh"]
    dtype = _DTYPES[case["dtype"]]
    s = {"lens": torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")}
    if case["kind"] == "append":
        n = case["n"]
        if case["source"] == "rows":
            s["k"], s["v"] = (_rows(g, (B, n, hk, dh)).to(dtype) for _ in range(2))
        elif case["source"] == "joint":
            joint = _rows(g, (B, n, 3 * hk, dh)).to(dtype)
            s["k"], s["v"] = joint[:, :, hk:2 * hk], joint[:, :, 2 * hk:]
        else:
            s["k"] = _rows(g, (B, n, hk, dh)).to(dtype).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            s["v"] = _rows(g, (B, n, hk, dh)).to(dtype).permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2)
        return s
    s["cache"] = _cache_inputs(case, g)
    if case["kind"] == "evict":
        k = case["k"]
        s["kept"] = torch.empty((B, k), dtype=torch.int32, device="cuda")
        for b, n in enumerate(_lengths(case)):
            order = torch.randperm(n, generator=g, device="cuda")[:min(k, n)].sort().values
            s["kept"][b, :order.numel()] = order.to(torch.int32)
            s["kept"][b, order.numel():] = -1                    # an image that has fewer rows than the list is long
        s["mass"] = torch.rand((B, case["kv_len"]), generator=g, device="cuda") ** 4
        return s
    H, n = case["heads"], case["n"]
    if case["packed_q"]:
        s["q"] = torch.randn((B, n, H + 2 * hk, dh), generator=g, device="cuda").to(dtype)[:, :, :H]
    else:
        s["q"] = torch.randn((B, n, H, dh), generator=g, device="cuda").to(dtype)
    if case["kind"] == "mass":
        s["lse"] = _attend_plain(case, s)[1]
        s["mass"] = torch.rand((B, case["kv_len"]), generator=g, device="cuda") ** 4
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _quantise(x):
    """Codes [..., dh / 2] and scale bytes [..., dh / 32] of rows [..., dh]."""
    x = x.float()
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    amax = y.abs().amax(-1)
    m, e = torch.frexp(amax)                                     # amax <= 6 2^e, e as small as that allows
    e = torch.where(m <= 0.75, e - 3, e - 2).clamp(-124, 125)
    e = torch.where(amax == 0, -124, e)
    bad = ~torch.isfinite(amax)
    z = torch.ldexp(y, -torch.where(bad, 0, e)[..., None])
    a = z.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() +
            (a >= 3.5).int() + (a > 5.0).int()) | (z < 0).int() * 8          # nearest; a tie goes to the even code
    code = torch.where(bad[..., None], 0, code).reshape(x.shape)
    codes = (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)
    return codes, torch.where(bad, 255, e + 127).to(torch.uint8)


def _values(codes, scales):
    """fp32 values [..., dh] of codes and scale bytes."""
    level = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], codes.shape[-1] * 2).int()
    v = level[code].reshape(*code.shape[:-1], code.shape[-1] // 32, 32)
    v = torch.ldexp(v, (scales.int() - 127)[..., None])
    return torch.where((scales == 255)[..., None], float("nan"), v).reshape(code.shape)


def _live(case, s):
    return torch.arange(case["kv_len"], device="cuda") < s["lens"][:, None]          # [B, L]


def _head_runs(case):
    """Runs of key heads whose scores and values are taken at once: as many as keep an intermediate tensor under 2 GiB."""
    B, n, dh, hk = case["B"], case["n"], case["dh"], case["kv_heads"]
    run = max(1, 2 ** 29 // (B * case["kv_len"] * max(case["heads"] // hk * n, dh)))
    return [slice(j, min(j + run, hk)) for j in range(0, hk, run)]


def _by_key_head(case, t):
    """[B, n, heads, ...] as [B, kv_heads, G n, ...]: the queries of the heads that share keys, head after head."""
    B, n, hk = case["B"], case["n"], case["kv_heads"]
    G = case["heads"] // hk
    return t.reshape(B, n, hk, G, -1).permute(0, 2, 3, 1, 4).reshape(B, hk, G * n, -1)


def _by_query(case, t):
    """The other way round."""
    B, n, hk = case["B"], case["n"], case["kv_heads"]
    return t.reshape(B, hk, case["heads"] // hk, n, -1).permute(0, 3, 1, 2, 4).reshape(B, n, case["heads"], -1)


def _scores(case, s, q, K):
    """Scores [B, heads of the run, G n, L]."""
    t = torch.matmul(q, K.transpose(2, 3)) / math.sqrt(case["dh"])
    return t.masked_fill(~_live(case, s)[:, None, None], float("-inf"))


def _attend_plain(case, s):
    kc, ks, vc, vs = s["cache"]
    q = _by_key_head(case, s["q"].float())
    live = _live(case, s)[:, None, :, None]
    outs, lses = [], []
    for r in _head_runs(case):
        t = _scores(case, s, q[:, r], _values(kc[:, r], ks[:, r]))
        top = t.amax(-1, keepdim=True)
        p = torch.exp(t - top)
        total = p.sum(-1, keepdim=True)
        V = torch.where(live, _values(vc[:, r], vs[:, r]), 0.0)
        outs.append(torch.matmul(p, V) / total)
        lses.append(top + torch.log(total))
    out = _by_query(case, torch.cat(outs, 1)).to(_DTYPES[case["dtype"]])
    return out, _by_query(case, torch.cat(lses, 1))[..., 0]


def _mass_plain(case, s):
    """Rows behind an image's length collect nothing and are marked -1."""
    kc, ks = s["cache"][:2]
    q, lse = _by_key_head(case, s["q"].float()), _by_key_head(case, s["lse"])
    total = 0.0
    for r in _head_runs(case):
        t = _scores(case, s, q[:, r], _values(kc[:, r], ks[:, r]))
        total = total + torch.exp(t - lse[:, r]).sum((1, 2))
    return torch.where(_live(case, s), s["mass"] + total, -1.0)


def _append_plain(case, s):
    out = []
    for x in (s["k"], s["v"]):
        codes, scales = _quantise(x)
        out.append(_values(codes, scales).to(_DTYPES[case["dtype"]]))
    return out


def _evict_plain(case, s):
    idx = s["kept"].long().clamp(min=0)
    have = s["kept"] >= 0                                        # [B, k]
    new = []
    for t in s["cache"]:
        pick = idx[:, None, :, None].expand(-1, t.shape[1], -1, t.shape[3])
        new.append(torch.gather(t, 2, pick))
    K, V = (torch.where(have[:, None, :, None], _values(*p), 0.0).permute(0, 2, 1, 3).to(torch.bfloat16)
            for p in (new[:2], new[2:]))
    mass = torch.where(have, torch.gather(s["mass"], 1, idx), -1.0)
    return K, V, mass, have.sum(1).to(torch.int32)


# ---- what is timed --------------------------------------------------------------------------------------------------
def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    global _NOVA
    from paper_2602_01345_amd import FourBitCache, Nova
    if _NOVA is None:
        _NOVA = Nova(0)
    B, hk, dh, dtype = case["B"], case["kv_heads"], case["dh"], _DTYPES[case["dtype"]]
    if case["kind"] == "append":
        n = case["n"]
        s["own"] = FourBitCache.empty(B, hk, case["kv_len"] + n, dh)
        # rows of images of one length are read back together; otherwise each image's own
        s["out"] = [torch.empty((B, n, hk, dh), dtype=dtype, device="cuda") for _ in range(2)]
        return
    s["own"] = FourBitCache(*s["cache"])
    if case["kind"] == "evict":
        s["dst"] = FourBitCache.empty(B, hk, case["k"], dh)
        s["mass_dst"] = torch.empty((B, case["k"]), device="cuda")
        s["lens_dst"] = torch.empty(B, dtype=torch.int32, device="cuda")
        s["out"] = [torch.empty((B, case["k"], hk, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        return
    H, n = case["heads"], case["n"]
    if case["kind"] == "attend":
        need = _NOVA.fourbit_attention_workspace_bytes(s["own"], H, n, case["kv_len"])
        s["out"] = torch.empty((B, n, H, dh), dtype=dtype, device="cuda")
        s["lse"] = torch.empty((B, n, H), device="cuda")
    else:
        s["lse"] = s["lse"].contiguous()                         # dense, as the attention call writes it
        need = _NOVA.fourbit_mass_workspace_bytes(s["own"], H, n, case["kv_len"])
        s["mass_out"] = torch.empty((B, case["kv_len"]), device="cuda")
    s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"append": _append_plain, "attend": _attend_plain, "mass": _mass_plain, "evict": _evict_plain}[kind](case, s)
    lens = s["lens"] if case["ragged"] else None
    if kind == "append":
        _NOVA.fourbit_append(s["own"], s["k"], s["v"], case["kv_len"], kv_len_per_row=lens)
        _NOVA.fourbit_unpack(s["own"], case["kv_len"], s["out"][0], s["out"][1], first_per_row=lens)
        return s["out"]
    if kind == "attend":
        _NOVA.fourbit_attention(s["own"], s["q"], s["out"], s["workspace"], case["kv_len"], lse=s["lse"], kv_len_per_row=lens)
        return s["out"], s["lse"]
    if kind == "mass":
        _NOVA.fourbit_mass(s["own"], s["q"], s["lse"], s["mass_out"], s["workspace"], case["kv_len"], mass_in=s["mass"],
                           kv_len_per_row=lens)
        return s["mass_out"]
    _NOVA.fourbit_evict(s["own"], s["dst"], s["kept"], case["kv_len"], kv_len_per_row=lens, kv_len_next=s["lens_dst"],
                        mass_src=s["mass"], mass_dst=s["mass_dst"])
    _NOVA.fourbit_unpack(s["dst"], 0, s["out"][0], s["out"][1], n_per_row=s["lens_dst"])
    return s["out"][0], s["out"][1], s["mass_dst"], s["lens_dst"]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _nearest64(x):
    """Values of rows in 4 bits: the nearest of the sixteen multiples of the group's scale, of two the one of even rank."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 6.0))
    e = torch.where(top <= 6.0 * torch.exp2(e - 1), e - 1, torch.where(top > 6.0 * torch.exp2(e), e + 1, e))
    step = torch.exp2(e.clamp(-124, 125))
    a = g.abs() / step
    best = torch.zeros_like(a)
    for rank in range(1, 8):
        half = (_LEVELS[rank - 1] + _LEVELS[rank]) / 2
        best = torch.where((a > half) | ((a == half) & (rank % 2 == 0)), _LEVELS[rank], best)
    return (torch.sign(g) * best * step).reshape(x.shape)


def _decode64(codes, scales):
    """float64 values of one cached tensor [n, dh / 2], [n, dh / 32]."""
    n = codes.shape[0]
    low, high = codes % 16, codes // 16
    c = torch.stack((low, high), 2).reshape(n, -1).to(torch.int64)
    mag, two = c % 8, c % 2
    exponent = torch.div(mag, 2, rounding_mode="floor")
    v = torch.where(exponent == 0, 0.5 * two.double(), (1 + 0.5 * two.double()) * torch.exp2(exponent.double() - 1))
    v = torch.where(c >= 8, -v, v)
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)


def exact(case, seed):
    s = _inputs(case, seed)
    B, hk, dh = case["B"], case["kv_heads"], case["dh"]
    if case["kind"] == "append":
        return [_nearest64(s["k"]), _nearest64(s["v"])]
    lens = _lengths(case)
    if case["kind"] == "evict":
        k = case["k"]
        K, V = (torch.zeros((B, k, hk, dh), dtype=torch.float64, device="cuda") for _ in range(2))
        mass = torch.full((B, k), -1.0, dtype=torch.float64, device="cuda")
        for b in range(B):
            n = min(k, lens[b])
            rows = s["kept"][b, :n].long()
            mass[b, :n] = s["mass"][b, rows].double()
            for j in range(hk):
                K[b, :n, j] = _decode64(s["cache"][0][b, j][rows], s["cache"][1][b, j][rows])
                V[b, :n, j] = _decode64(s["cache"][2][b, j][rows], s["cache"][3][b, j][rows])
        return K, V, mass, torch.tensor([min(k, n) for n in lens], dtype=torch.int32, device="cuda")
    H, n = case["heads"], case["n"]
    G = H // hk
    out = torch.zeros((B, n, H, dh), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, n, H), dtype=torch.float64, device="cuda")
    mass = torch.full((B, case["kv_len"]), -1.0, dtype=torch.float64, device="cuda")
    for b in range(B):
        L = lens[b]
        if case["kind"] == "mass":
            mass[b, :L] = s["mass"][b, :L].double()
        for j in range(hk):
            K = _decode64(s["cache"][0][b, j, :L], s["cache"][1][b, j, :L])
            V = _decode64(s["cache"][2][b, j, :L], s["cache"][3][b, j, :L]) if case["kind"] == "attend" else None
            for h in range(j * G, (j + 1) * G):
                t = s["q"][b, :, h].double() @ K.T.contiguous() / math.sqrt(dh)
                if case["kind"] == "mass":
                    mass[b, :L] += torch.exp(t - s["lse"][b, :, h].double()[:, None]).sum(0)
                else:
                    lse[b, :, h] = torch.logsumexp(t, 1)
                    out[b, :, h] = torch.softmax(t, 1) @ V
    return mass if case["kind"] == "mass" else (out, lse)
