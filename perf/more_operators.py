"""Operators on a key/value cache in pages: what is measured of them, and their plain forms.

A pool holds K and V as pages [pages, kv_heads, p, dh] of p rows; image b's row j lies in page table[b, j // p], row j % p.

  reserve  page lists and slot maps from the images' lengths: images give up rows, then new ones come; pages come from and go
           to a stack of free ones; the slot of a row is its page times p plus its row there, -1 where there is none
  append   rows to their slots
  attend   attention of a chunk of n queries per image, the last n rows of the image, over all of its rows or (causal) those up to
           the query's own; with the logarithm of each softmax sum
  choose   summaries of the pages the last n rows lie in (mean keys, rounded to 7 bits under the largest channel of the page), then
           the k pages that score highest for each query: first and last visible page, and the best products of the query,
           rounded likewise, and the summary, largest over the heads that share a key head
  sparse   attention over the rows of chosen pages alone

Sizes are those of this repository's workloads (256- to 1024-pixel scale lists) and generic ones for serving.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZES = {"f32": 4, "bf16": 2}
_NOVA = None


# ---- the cases ------------------------------------------------------------------------------------------------------
def _reserve(name, B, page_rows, n, kv_len, turnover, short=False):
    return {"name": name, "kind": "reserve", "B": B, "page_rows": page_rows, "n": n, "kv_len": kv_len, "turnover": turnover,
            "short": short, "ragged": True}


def _append(name, dtype, B, kv_heads, dh, n, kv_len, page_rows, source, ragged=False):
    return {"name": name, "kind": "append", "dtype": dtype, "B": B, "kv_heads": kv_heads, "dh": dh, "n": n, "kv_len": kv_len,
            "page_rows": page_rows, "source": source, "ragged": ragged}


def _query(name, kind, dtype, B, heads, kv_heads, dh, n, kv_len, page_rows, causal=False, ragged=False, packed_q=False, k=0):
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "heads": heads, "kv_heads": kv_heads, "dh": dh, "n": n,
            "kv_len": kv_len, "page_rows": page_rows, "causal": causal, "ragged": ragged, "packed_q": packed_q, "k": k}


def listed():
    return [
        # every request of a large batch gets one more token; a sixteenth of them needs a new page
        _reserve("reserve-token-b256", 256, 16, 1, 4096, turnover=False),
        # prompts of different lengths come in, a part of them in the place of requests that are done
        _reserve("reserve-prompts-b64", 64, 64, 2048, 8192, turnover=True),
        # one new row per request: the least there is to append
        _append("append-token-b64", "bf16", 64, 8, 128, 1, 2048, 16, "rows", ragged=True),
        # all tokens of the last scale of two 1024-pixel images, as they lie in the output of a joint projection
        _append("append-1024px-b2", "bf16", 2, 16, 128, 4096, 6425, 64, "joint"),
        # a handful of fp32 queries against all rows before the scale 40 x 40: the smallest attention, latency
        _query("attend-few-f32", "attend", "f32", 2, 16, 16, 64, 5, 2521, 16, packed_q=True),
        # token by token over long caches of different lengths, four query heads to a key head, small pages
        _query("attend-token-32k", "attend", "bf16", 4, 32, 8, 128, 1, 32768, 16, ragged=True),
        # last scale of 512-pixel images, half of the tokens kept, images of different lengths, 36 heads
        _query("attend-512px-b8", "attend", "bf16", 8, 36, 36, 64, 512, 1728, 32, ragged=True),
        # a chunk of two long prompts behind what they have in the cache: the largest
        _query("attend-chunk-16k", "attend", "bf16", 2, 32, 8, 128, 2048, 16384, 64, causal=True),
        # one token per request chooses its pages of a long cache
        _query("choose-token-32k", "choose", "bf16", 4, 32, 8, 128, 1, 32768, 64, ragged=True, k=32),
        # every token of a chunk chooses for itself
        _query("choose-chunk-32k", "choose", "bf16", 1, 32, 8, 128, 1024, 32768, 64, causal=True, k=32),
        # one token per request over what it has chosen of a very long cache
        _query("sparse-token-128k", "sparse", "bf16", 4, 32, 8, 128, 1, 131072, 64, ragged=True, k=64),
        # a chunk whose tokens have chosen a sixteenth of their cache each
        _query("sparse-chunk-32k", "sparse", "bf16", 1, 32, 8, 128, 1024, 32768, 64, causal=True, k=32),
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
        kind = rng.choice(("reserve", "append", "attend", "attend", "attend", "choose", "choose", "sparse", "sparse"))
        page_rows = rng.choice((16, 32, 64, 128, 256))
        ragged = rng.random() < 0.5
        if kind == "reserve":
            return {"kind": kind, "B": _log_int(rng, 1, 512), "page_rows": page_rows, "n": _log_int(rng, 1, 4096),
                    "kv_len": _log_int(rng, 1, 32768), "turnover": rng.random() < 0.5, "short": rng.random() < 0.3, "ragged": True}
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        dh = rng.choice((64, 128))
        kv_heads = _log_int(rng, 1, 36)
        B = _log_int(rng, 1, 16)
        n = 1 if rng.random() < 0.3 else _log_int(rng, 1, 2048)
        kv_len = n + _log_int(rng, 1, 32768) - 1
        case = {"kind": kind, "dtype": dtype, "B": B, "kv_heads": kv_heads, "dh": dh, "n": n, "kv_len": kv_len,
                "page_rows": page_rows, "ragged": ragged}
        if kind == "append":
            case["source"] = rng.choice(("rows", "joint", "caches"))
        else:
            pages = -(-kv_len // page_rows)
            # a page list as long as it makes sense for a cache of this length: from two to a quarter of the pages, 128 at most
            case.update(heads=kv_heads * rng.choice((1, 1, 2, 3, 4, 8)), causal=rng.random() < 0.5, packed_q=rng.random() < 0.3,
                        k=0 if kind == "attend" else rng.randint(2, max(2, min(128, pages // 4))))
        # what the pool, or the scores of one key head of an image, take
        rows = B * (kv_len + n + page_rows) * kv_heads * dh
        if _cost(case) <= most and rows <= 2 ** 30:
            return case


def _visible_pairs(case):
    """(query, key) pairs of one head that count."""
    n, k, p = case["n"], case["k"], case["page_rows"]
    total = 0
    for L in _lengths(case):
        if not k:
            total += n * L - (n * (n - 1) // 2 if case["causal"] else 0)
        else:
            total += sum(min(L - n + s + 1 if case["causal"] else L, k * p) for s in range(n))
    return total


def work(case):
    B, n, p = case["B"], case["n"], case["page_rows"]
    kind = case["kind"]
    if kind == "reserve":
        return {"bytes": B * (n + 4) * 4 + B * 8 * -(-n // p), "flops": 0}
    hk, dh, e = case["kv_heads"], case["dh"], _SIZES[case["dtype"]]
    if kind == "append":
        return {"bytes": 2 * 2 * B * n * hk * dh * e + 4 * B * n, "flops": 0}
    H, k = case["heads"], case["k"]
    q = B * n * H * dh * e
    if kind == "choose":
        pages = sum(-(-L // p) for L in _lengths(case))
        means = pages * hk * dh * 2
        return {"bytes": q + means + B * n * hk * k * 4 + B * n * hk * dh * e, "flops": 2 * n * H * pages * dh}
    rows = sum(_lengths(case))
    if kind == "sparse":                                         # the pages of one query: others may have chosen the same
        rows = sum(min(L, k * p) for L in _lengths(case))
    chosen = B * n * hk * k * 4
    return {"bytes": 2 * rows * hk * dh * e + 2 * q + B * n * H * 4 + chosen, "flops": 4 * H * dh * _visible_pairs(case)}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Rows every image has.  "ragged": from the full length down to a quarter of it, spread evenly, n at least (queries are rows
    of their image; for appends and reservations the n rows come on top)."""
    B, L, n = case["B"], case["kv_len"], case["n"]
    if not case["ragged"]:
        return [L] * B
    least = n if case["kind"] in ("attend", "choose", "sparse") else 0
    return [max(L - (3 * L * b) // (4 * B), least) for b in range(B)]


def _counts(case):
    """Rows that come to every image of a reservation: all different, none for some."""
    B, n = case["B"], case["n"]
    return [n - (n * ((b * 7) % B)) // B for b in range(B)]


def _kept(case):
    """Rows every image of a reservation keeps: with turnover every fourth has been replaced by another, every eighth cut back."""
    return [L if not case["turnover"] or b % 4 < 2 else L // 2 if b % 8 == 2 else 0 for b, L in enumerate(_lengths(case))]


def _ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _page_lists(case, g, pitch, extra):
    """A page table [B, pitch] of a pool whose pages are in no order, -1 behind an image's pages; how many pages the pool has, and
    those that nobody has."""
    p = case["page_rows"]
    counts = [-(-L // p) for L in _lengths(case)]
    pages = sum(counts) + extra
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    have = torch.arange(pitch, device="cuda") < torch.tensor(counts, device="cuda")[:, None]
    table = torch.full((case["B"], pitch), -1, dtype=torch.int32, device="cuda")
    table[have] = order[:sum(counts)]
    return table, pages, order[sum(counts):]


def _tokens(g, B, n, heads, dh):
    """fp32 rows [B, n, heads, dh] of neighbouring tokens: runs of 64 share a part, channels have different reach."""
    reach = torch.exp(0.5 * torch.randn((heads, dh), generator=g, device="cuda"))
    run = torch.randn((B, -(-n // 64), heads, dh), generator=g, device="cuda").repeat_interleave(64, 1)[:, :n]
    return (0.7 * run + 0.7 * torch.randn((B, n, heads, dh), generator=g, device="cuda")) * reach


def _pool(case, g, s, rows):
    """Pools of K and V with these many rows [B] of every image; whatever else lies in them is left as memory may hold it: NaN, or
    numbers where the pools are outputs."""
    B, hk, dh, p = case["B"], case["kv_heads"], case["dh"], case["page_rows"]
    dtype = _DTYPES[case["dtype"]]
    rest = 7.0 if case["kind"] == "append" else float("nan")
    pools = []
    for _ in range(2):
        pool = torch.full((s["pages"], hk, p, dh), rest, dtype=dtype, device="cuda")
        for b, L in enumerate(rows):
            if L == 0:
                continue
            m = -(-L // p)
            x = torch.full((m * p, hk, dh), rest, dtype=dtype, device="cuda")
            x[:L] = _tokens(g, 1, L, hk, dh)[0].to(dtype)
            pool[s["table"][b, :m].long()] = x.reshape(m, p, hk, dh).permute(0, 2, 1, 3)
        pools.append(pool)
    return pools


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, n, p, L = case["B"], case["n"], case["page_rows"], case["kv_len"]
    lens = _lengths(case)
    s = {"lens": _ints(lens)}
    if case["kind"] == "reserve":
        counts, kept = _counts(case), _kept(case)
        need = sum(max(-(-(k + c) // p) - -(-a // p), 0) for a, k, c in zip(lens, kept, counts))
        table, pages, free = _page_lists(case, g, -(-(L + n) // p), need // 2 if case["short"] else need + 5)
        s.update(table=table, pages=pages, counts=_ints(counts), kept=_ints(kept), free_count=_ints([free.numel()]))
        s["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        s["free"][:free.numel()] = free
        return s
    hk, dh = case["kv_heads"], case["dh"]
    dtype = _DTYPES[case["dtype"]]
    if case["kind"] == "append":
        after = dict(case, kv_len=L + n, ragged=False)
        s["table"], s["pages"], _ = _page_lists(after, g, -(-(L + n) // p), 3)
        s["cache"] = _pool(case, g, s, lens)
        at = s["lens"][:, None] + torch.arange(n, device="cuda")                          # [B, n]
        s["slots"] = (torch.gather(s["table"], 1, at // p) * p + at % p).to(torch.int32)
        if case["source"] == "joint":
            joint = _tokens(g, B, n, 3 * hk, dh).to(dtype)
            s["k"], s["v"] = joint[:, :, hk:2 * hk], joint[:, :, 2 * hk:]
        else:
            s["k"], s["v"] = (_tokens(g, B, n, hk, dh).to(dtype) for _ in range(2))
        if case["source"] == "caches":                           # the dense layouts: keys by row, values key-minor
            s["k"] = s["k"].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            s["v"] = s["v"].permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2)
        return s
    s["table"], s["pages"], _ = _page_lists(case, g, -(-L // p) + 1, 3)
    s["cache"] = _pool(case, g, s, lens)
    H = case["heads"]
    q = _tokens(g, B, n, H + 2 * hk if case["packed_q"] else H, dh).to(dtype)
    s["q"] = q[:, :, :H]
    if case["kind"] != "attend":
        s["means"] = torch.zeros((s["pages"], hk, dh), dtype=torch.bfloat16, device="cuda")
        _summarise_plain(case, s, [0] * B)
    if case["kind"] == "sparse":
        s["chosen"] = _choose_plain(case, s)
    if case["kind"] == "choose":                                 # the pages of the last n rows are still to be summarised
        for b, have in enumerate(lens):
            s["means"][s["table"][b, (have - n) // p:-(-have // p)].long()] = 1.0
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e as float64, exactly, for whole numbers e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _seven_bits(x, dims):
    """float64 x as whole multiples of a power of two, 127 of them at most; one power for all of `dims`.  Returns both."""
    top = x.abs().amax(dims, keepdim=True)
    m, e = torch.frexp(top)                                      # top <= 127 2^e, e as small as that allows
    e = torch.where(m <= 127 / 128, e - 7, e - 6)
    e = torch.where(top == 0, -100, e).clamp(-100, 100)
    return torch.round(x * _two_to(-e)).clamp(-127, 127), e


def _summarise_plain(case, s, first):
    """Means of the pages that the rows from first[b] on lie in, written into s["means"]."""
    p, table = case["page_rows"], s["table"]
    for b, L in enumerate(_lengths(case)):
        a, z = first[b] // p, -(-L // p)
        pages = table[b, a:z].long()
        rows = torch.arange(a * p, z * p, device="cuda").reshape(-1, 1, p, 1)
        x = torch.where(rows < L, s["cache"][0][pages].double(), 0.0)
        count = (rows < L).sum(2).double()                       # [pages, 1, 1]
        w, e = _seven_bits(x.sum(2) / count, -1)
        s["means"][pages] = (w * _two_to(e)).to(torch.bfloat16)


def _visible(case, s):
    """Keys that query s of image b sees, [B, n]."""
    n = case["n"]
    at = torch.arange(1, n + 1, device="cuda") - n if case["causal"] else torch.zeros(n, dtype=torch.long, device="cuda")
    return (s["lens"].long()[:, None] + at).clamp(min=0)


def _by_key_head(case, t):
    """[n, heads, dh] of one image as [kv_heads, G n, dh]: the queries of the heads that share keys, head after head."""
    hk = case["kv_heads"]
    return t.reshape(case["n"], hk, case["heads"] // hk, -1).permute(1, 2, 0, 3).reshape(hk, -1, t.shape[-1])


def _by_query(case, t):
    """The other way round."""
    hk = case["kv_heads"]
    return t.reshape(hk, case["heads"] // hk, case["n"], -1).permute(2, 0, 1, 3).reshape(case["n"], case["heads"], -1)


def _choose_plain(case, s):
    B, n, hk, p, k = case["B"], case["n"], case["kv_heads"], case["page_rows"], case["k"]
    G, P = case["heads"] // hk, s["table"].shape[1]
    chosen = torch.empty((B, n, hk, k), dtype=torch.int32, device="cuda")
    vis = -(-_visible(case, s) // p)                             # pages that are seen, [B, n]
    i = torch.arange(P, device="cuda")
    for b in range(B):
        means = s["means"][s["table"][b].long().clamp(min=0)].float().permute(1, 2, 0).contiguous()       # [hk, dh, P]
        w, _ = _seven_bits(s["q"][b].double().reshape(n, hk, G, -1), (2, 3))
        # whole numbers under 2^21 times one power of two: exact in 32 bits
        score = torch.matmul(_by_key_head(case, w.float()), means).reshape(hk, G, n, P).amax(1)
        v = vis[b][:, None]
        score = torch.where((i == 0) | (i == v - 1) | score.isnan(), float("inf"), score)
        score = torch.where(i < v, score, float("-inf"))
        order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :k]                  # [hk, n, k]
        if P < k:
            order = torch.cat((order, torch.full((hk, n, k - P), P, device="cuda")), -1)
        order = torch.where(order < v, order, P).sort(-1).values
        chosen[b] = torch.where(order < P, order, -1).to(torch.int32).permute(1, 0, 2)
    return chosen


def _attend_plain(case, s, chosen=None):
    B, n, H, hk, dh, p = (case[x] for x in ("B", "n", "heads", "kv_heads", "dh", "page_rows"))
    G = H // hk
    out = torch.empty((B, n, H, dh), dtype=_DTYPES[case["dtype"]], device="cuda")
    lse = torch.empty((B, n, H), device="cuda")
    vis = _visible(case, s)
    for b, L in enumerate(_lengths(case)):
        m = -(-L // p)
        pages = s["table"][b, :m].long()
        q = _by_key_head(case, s["q"][b].float())
        dead = (torch.arange(L, device="cuda") >= vis[b][:, None])[None]                  # [1 or hk, n, L]
        if chosen is not None:
            c = chosen[b].long().permute(1, 0, 2)
            take = torch.zeros((hk, n, m + 1), dtype=torch.bool, device="cuda")
            take.scatter_(2, torch.where((c >= 0) & (c < m), c, m), True)
            dead = dead | ~take[..., :m].repeat_interleave(p, 2)[..., :L]
        outs, lses = [], []
        run = max(1, 2 ** 28 // (L * max(G * n, dh)))            # key heads whose scores are taken at once: up to 1 GiB of them
        for j in range(0, hk, run):
            K, V = (c[pages, j:j + run].permute(1, 0, 2, 3).reshape(-1, m * p, dh)[:, :L].float() for c in s["cache"])
            t = torch.matmul(q[j:j + run], K.transpose(1, 2).contiguous()) / math.sqrt(dh)
            gone = dead if chosen is None else dead[j:j + run]
            t = t.reshape(-1, G, n, L).masked_fill(gone[:, None], float("-inf")).reshape(-1, G * n, L)
            top = t.amax(-1, keepdim=True)
            e = torch.exp(t - top)
            total = e.sum(-1, keepdim=True)
            outs.append(torch.matmul(e, V) / total)
            lses.append(top + torch.log(total))
        out[b] = _by_query(case, torch.cat(outs)).to(out.dtype)
        lse[b] = _by_query(case, torch.cat(lses))[..., 0]
    return out, lse


def _append_plain(case, s):
    p = case["page_rows"]
    slots = s["slots"].long()
    for pool, x in zip(s["cache"], (s["k"], s["v"])):
        pool[slots // p, :, slots % p] = x                       # [B, n, hk, dh]
    return s["cache"]


def _reserve_plain(case, s):
    B, n, p = case["B"], case["n"], case["page_rows"]
    table, free, pages, P = s["table"].clone(), s["free"].clone(), s["pages"], s["table"].shape[1]
    now, keep, count = s["lens"].long(), s["kept"].long(), s["counts"].long()
    keep = torch.minimum(keep, now)
    held, want = -(-now // p), -(-(keep + count) // p)
    less, more = (held - want).clamp(min=0), (want - held).clamp(min=0)
    stack = s["free_count"].long()
    # released pages, in the order of images and pages, go onto the stack
    i = torch.arange(P, device="cuda")
    gone = (i >= want[:, None]) & (i < held[:, None])
    rank = (less.cumsum(0) - less)[:, None] + i - want[:, None]
    released = torch.full((pages + 1,), -1, dtype=torch.int32, device="cuda")
    released[torch.where(gone, rank, pages)] = torch.where(gone, table, -1)
    height = stack + less.sum()
    served = more.cumsum(0) <= height
    more = torch.where(served, more, 0)
    # and images that grow take theirs from its top
    comes = (i >= held[:, None]) & (i < (held + more)[:, None])
    at = height - 1 - ((more.cumsum(0) - more)[:, None] + i - held[:, None])
    page = torch.where(at >= stack, released[(at - stack).clamp(0, pages)], free[at.clamp(0, pages - 1)])
    table = torch.where(comes, page, table)
    left = height - more.sum()
    at = torch.arange(pages, device="cuda")
    free = torch.where((at >= stack) & (at < left), released[(at - stack).clamp(0, pages)], free)
    after = torch.where(served | (want <= held), keep + count, torch.minimum(keep + count, held * p))
    row = keep[:, None] + torch.arange(n, device="cuda")
    slots = torch.gather(table, 1, (row // p).clamp(max=P - 1)) * p + row % p
    slots = torch.where(row < after[:, None], slots, -1).to(torch.int32)
    return table, slots, after.to(torch.int32), free, left.to(torch.int32)


# ---- what is timed --------------------------------------------------------------------------------------------------
def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    global _NOVA
    from paper_2602_01345_amd import Nova, PagedCache
    if _NOVA is None:
        _NOVA = Nova(0)
    B, n = case["B"], case["n"]
    if case["kind"] == "reserve":
        s["slots"] = torch.empty((B, n), dtype=torch.int32, device="cuda")
        s["lens_next"] = torch.empty(B, dtype=torch.int32, device="cuda")
        s["free_next"] = torch.empty(1, dtype=torch.int32, device="cuda")
        return
    s["own"] = PagedCache(*s["cache"])
    if case["kind"] == "append":
        return
    H, hk = case["heads"], case["kv_heads"]
    if case["kind"] == "choose":
        s["idx"] = torch.empty((B, n, hk, case["k"]), dtype=torch.int32, device="cuda")
        return
    if case["kind"] == "attend":
        need = _NOVA.paged_attention_workspace_bytes(s["own"], B, H, n, case["kv_len"])
    else:
        need = _NOVA.paged_sparse_attention_workspace_bytes(s["own"], B, H, n, case["kv_len"], case["k"])
    s["out"] = torch.empty((B, n, H, case["dh"]), dtype=_DTYPES[case["dtype"]], device="cuda")
    s["lse"] = torch.empty((B, n, H), device="cuda")
    s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "choose":
            _summarise_plain(case, s, [L - case["n"] for L in _lengths(case)])
            return s["means"], _choose_plain(case, s)
        if kind == "sparse":
            return _attend_plain(case, s, s["chosen"])
        return {"reserve": _reserve_plain, "append": _append_plain, "attend": _attend_plain}[kind](case, s)
    L = case["kv_len"]
    if kind == "reserve":
        _NOVA.paged_reserve(s["table"], case["page_rows"], case["n"], L, s["free"], s["free_count"], s["lens_next"],
                            s["free_next"], slots=s["slots"], kv_len_per_row=s["lens"], n_per_row=s["counts"],
                            keep_per_row=s["kept"])
        return s["table"], s["slots"], s["lens_next"], s["free"], s["free_next"]
    if kind == "append":
        _NOVA.paged_append(s["own"], s["k"], s["v"], s["slots"])
        return s["cache"]
    lens = s["lens"] if case["ragged"] else None
    if kind == "choose":
        _NOVA.paged_summarise(s["own"], s["table"], s["means"], case["n"], L, kv_len_per_row=lens)
        _NOVA.paged_select(s["means"], s["table"], case["page_rows"], s["q"], s["idx"], L, first=1, recent=1,
                           causal=case["causal"], kv_len_per_row=lens)
        return s["means"], s["idx"]
    if kind == "attend":
        _NOVA.paged_attention(s["own"], s["table"], s["q"], s["out"], s["workspace"], L, causal=case["causal"], lse=s["lse"],
                              kv_len_per_row=lens)
    else:
        _NOVA.paged_sparse_attention(s["own"], s["table"], s["chosen"], s["q"], s["out"], s["workspace"], L,
                                     causal=case["causal"], lse=s["lse"], kv_len_per_row=lens)
    return s["out"], s["lse"]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _exact_reserve(case, s):
    p, n = case["page_rows"], case["n"]
    table, free = s["table"].tolist(), s["free"].tolist()
    stack = free[:s["free_count"].item()]
    now, keep, counts = _lengths(case), _kept(case), _counts(case)
    after, slots = [], []
    for b in range(case["B"]):
        for i in range(math.ceil((keep[b] + counts[b]) / p), math.ceil(now[b] / p)):
            stack.append(table[b][i])
    out_of_pages = False
    for b in range(case["B"]):
        held, want = math.ceil(now[b] / p), math.ceil((keep[b] + counts[b]) / p)
        rows = keep[b] + counts[b]
        if want > held:
            out_of_pages = out_of_pages or want - held > len(stack)
            if out_of_pages:
                rows = min(rows, held * p)
            else:
                for i in range(held, want):
                    table[b][i] = stack.pop()
        after.append(rows)
        slots.append([table[b][r // p] * p + r % p if r < rows else -1 for r in range(keep[b], keep[b] + n)])
    # what lies above the stack stays as it was
    free = stack + free[len(stack):]
    return _ints(table), _ints(slots), _ints(after), _ints(free), _ints([len(stack)])


def _image_rows(case, s, b, which, j):
    """float64 rows of image b, key head j, one after the other."""
    L, p = _lengths(case)[b], case["page_rows"]
    r = torch.arange(L, device="cuda")
    return s["cache"][which][s["table"][b][r // p].long(), j, r % p].double()


def _exact_means(case, s):
    n, p, hk = case["n"], case["page_rows"], case["kv_heads"]
    means = s["means"].double()
    for b, L in enumerate(_lengths(case)):
        a = (L - n) // p * p
        group = torch.arange(L - a, device="cuda") // p
        count = torch.bincount(group).double()[:, None]
        for j in range(hk):
            x = _image_rows(case, s, b, 0, j)[a:]
            total = torch.zeros((count.shape[0], x.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, group, x)
            means[s["table"][b, a // p:a // p + count.shape[0]].long(), j] = _nearest_seven(total / count)
    return means


def _nearest_seven(x):
    """Rows of x as the nearest multiples (of two the even one) of the smallest power of two of which 127 reach the row's largest."""
    top = x.abs().amax(-1, keepdim=True).cpu()
    e = torch.full_like(top, -100.0)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):                   # the smallest e >= -100 that reaches, bit by bit from below
        e = torch.where(top > 127 * 2.0 ** (e + step - 1), e + step, e)
    unit = (2.0 ** e.clamp(max=100)).to(x.device)
    return torch.round(x / unit).clamp(-127, 127) * unit


def _exact_choose(case, s):
    import numpy as np
    B, n, hk, p, k = case["B"], case["n"], case["kv_heads"], case["page_rows"], case["k"]
    G = case["heads"] // hk
    means = _exact_means(case, s)
    chosen = np.full((B, n, hk, k), -1, dtype=np.int64)
    for b, L in enumerate(_lengths(case)):
        P = math.ceil(L / p)
        seen = np.array([L - n + t + 1 if case["causal"] else L for t in range(n)])
        pages = np.ceil(seen / p).astype(np.int64)[:, None]
        for j in range(hk):
            m = means[s["table"][b, :P].long(), j]
            q = _nearest_seven(s["q"][b, :, j * G:(j + 1) * G].double().reshape(n, -1)).reshape(n, G, -1)
            score = torch.stack([q[:, h] @ m.T.contiguous() for h in range(G)]).amax(0).cpu().numpy()
            i = np.arange(P)
            score[(i == 0) | (i == pages - 1)] = np.inf
            score = np.where(i < pages, score, -np.inf)
            best = np.argsort(-score, axis=1, kind="stable")[:, :k]
            best = np.sort(np.where(best < pages, best, P), axis=1)
            chosen[b, :, j, :best.shape[1]] = np.where(best < P, best, -1)
    return means, torch.from_numpy(chosen).to(torch.int32).cuda()


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "reserve":
        return _exact_reserve(case, s)
    B, n, hk, dh, p = case["B"], case["n"], case["kv_heads"], case["dh"], case["page_rows"]
    if kind == "append":
        pools = [t.double() for t in s["cache"]]
        for pool, x in zip(pools, (s["k"], s["v"])):
            flat = pool.permute(0, 2, 1, 3).reshape(-1, hk, dh).clone()
            flat[s["slots"].long().flatten()] = x.reshape(-1, hk, dh).double()
            pool.copy_(flat.reshape(-1, p, hk, dh).permute(0, 2, 1, 3))
        return pools
    if kind == "choose":
        return _exact_choose(case, s)
    H = case["heads"]
    G = H // hk
    out = torch.zeros((B, n, H, dh), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, n, H), dtype=torch.float64, device="cuda")
    for b, L in enumerate(_lengths(case)):
        r = torch.arange(L, device="cuda")
        last = torch.arange(L - n, L, device="cuda")[:, None] if case["causal"] else L - 1
        for j in range(hk):
            K, V = (_image_rows(case, s, b, w, j) for w in range(2))
            counts = (r <= last).expand(n, L)
            if kind == "sparse":
                member = torch.zeros((n, s["table"].shape[1] + 1), dtype=torch.bool, device="cuda")
                member.scatter_(1, s["chosen"][b, :, j].long() % member.shape[1], True)          # -1: the column behind all pages
                counts = counts & member[:, r // p]
            for h in range(j * G, (j + 1) * G):
                t = (s["q"][b, :, h].double() @ K.T.contiguous() / math.sqrt(dh)).masked_fill(~counts, -math.inf)
                lse[b, :, h] = torch.logsumexp(t, 1)
                out[b, :, h] = torch.softmax(t, 1) @ V
    return out, lse
