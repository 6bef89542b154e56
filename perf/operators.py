"""Attention with a sliding window and sinks, and eviction from the paged cache by accumulated attention weight, as cases that can be
timed and compared: once in plain torch, once through the public calls of paper_2609_33135_b200.binding.

  window_prompt   mpfa_prefill_window: a whole prompt, each query sees the last `window` keys and the first `sinks`
  window_chunk    mpfa_prefill_paged_window: a chunk of queries per request against the pages; pages out of everyone's view are gone
  window_decode   mpfa_decode_window: one query token per request; pages out of view are gone
  weights_decode  mpfa_decode_weights: one query token per request over its whole context, and what each key received of its attention
                  added to the key's running sum
  evict           mpfa_evict_paged: the sinks, the newest tokens and the heaviest of the others of each kv head move to new pages

The operands are the library's: Q and K as NVFP4 (two E2M1 codes a byte, an E4M3 scale for 16 channels, a tensor scale), V as E4M3, the
compensation vector Delta_S in BF16, in the layouts of include/mpfa.h.  Arithmetic of attention as the method defines it: logits in
FP32, softmax over 128-key blocks from the last to the first with a running maximum, P as E4M3(448 P), everything else in FP32.
"""
import math
import random

import torch

own = False

D = 128
PAGE = 64
TILE = 128
PART = 8   # blocks of a decode partition
LOG2E = 1.4426950408889634


def listed():
    return [
        # a short prompt of a small model with a narrow window: launches and latency
        _prompt("window_prompt_short", 1, 300, 8, 2, 128, 4),
        # an ordinary prompt, ragged, a window of a quarter of it
        _prompt("window_prompt_4k", 1, 4001, 32, 8, 1024, 4),
        # several prompts on the 40:8 shape, odd window, more sinks than a block
        _prompt("window_prompt_batch", 3, 1999, 40, 8, 700, 130),
        # the benchmark's long prompt under a wide window
        _prompt("window_prompt_16k", 1, 16384, 32, 8, 4096, 64),
        # chunked prefill: four requests, 512 new tokens each on ragged contexts of which the window is left
        {"name": "window_chunk_512", "kind": "window_chunk", "B": 4, "N_q": 512, "len_lo": 2000, "len_hi": 16000, "H_q": 32, "H_kv": 8,
         "window": 2048, "sinks": 4},
        # interactive decoding of one request: latency
        _decode("window_decode_single", 1, 5000, 5000, 32, 8, 1024, 4),
        # a chat server's batch, contexts shorter and longer than the window, odd window
        _decode("window_decode_batch", 64, 100, 40000, 40, 8, 4095, 4),
        # a long-context batch under a wide window: bound by reading the cache
        _decode("window_decode_wide", 32, 16384, 131072, 32, 8, 16384, 128),
        # interactive decoding that keeps account of the weights: latency
        dict(_decode("weights_decode_single", 1, 4097, 4097, 32, 8, 0, 0), kind="weights_decode"),
        # a batch of contexts around an eviction budget of 4096 tokens, ragged
        dict(_decode("weights_decode_batch", 64, 1000, 8192, 40, 8, 0, 0), kind="weights_decode"),
        # one request that has outgrown its budget
        _evict("evict_single", 1, 4608, 4608, 32, 8, 4096, 4, 256),
        # a batch cut back to its budget, ragged lengths, an odd budget
        _evict("evict_batch", 32, 4200, 9000, 32, 8, 4001, 4, 1000),
    ]


def _prompt(name, B, N, H_q, H_kv, window, sinks):
    return {"name": name, "kind": "window_prompt", "B": B, "N": N, "H_q": H_q, "H_kv": H_kv, "window": window, "sinks": sinks}


def _decode(name, B, len_lo, len_hi, H_q, H_kv, window, sinks):
    return {"name": name, "kind": "window_decode", "B": B, "len_lo": len_lo, "len_hi": len_hi, "H_q": H_q, "H_kv": H_kv,
            "window": window, "sinks": sinks}


def _evict(name, B, len_lo, len_hi, H_q, H_kv, keep, sinks, recent):
    return {"name": name, "kind": "evict", "B": B, "len_lo": len_lo, "len_hi": len_hi, "H_q": H_q, "H_kv": H_kv, "keep": keep,
            "sinks": sinks, "recent": recent}


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of these ranges: contexts of 1 to 131072 tokens, windows of 1 to 16384, 0 to 300 sinks, groups of 1 to 8 heads."""
    H_q, H_kv = rng.choice(((4, 4), (8, 2), (8, 1), (16, 16), (32, 8), (32, 8), (40, 8)))
    kind = rng.choice(("window_prompt", "window_chunk", "window_decode", "weights_decode", "evict"))
    sinks = rng.choice((0, 1, 4, 4, 64, 130, 300))
    top = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("window_prompt", "window_decode", "weights_decode", "evict")}
    while True:
        if kind == "window_prompt":
            c = _prompt("", _log_int(rng, 1, 8), _log_int(rng, 1, 16384), H_q, H_kv, _log_int(rng, 1, 8192), sinks)
        elif kind == "window_chunk":
            B, N_q, hi = _log_int(rng, 1, 8), _log_int(rng, 1, 2048), _log_int(rng, 64, 65536)
            if hi <= N_q:
                continue
            c = {"kind": kind, "B": B, "N_q": N_q, "len_lo": _log_int(rng, N_q + 1, hi), "len_hi": hi, "H_q": H_q, "H_kv": H_kv,
                 "window": _log_int(rng, 1, 8192), "sinks": sinks}
        elif kind in ("window_decode", "weights_decode"):
            B, hi = _log_int(rng, 1, 256), _log_int(rng, 16, 131072 if kind == "window_decode" else 32768)
            c = dict(_decode("", B, _log_int(rng, 1, hi), hi, H_q, H_kv, _log_int(rng, 1, 16384), sinks), kind=kind)
            if kind == "weights_decode":
                c["window"] = c["sinks"] = 0
        else:
            B, hi = _log_int(rng, 1, 64), _log_int(rng, 64, 65536)
            keep = _log_int(rng, 32, hi)
            sinks = min(sinks, keep // 4)
            c = _evict("", B, _log_int(rng, max(1, keep // 2), hi), hi, H_q, H_kv, keep, sinks, rng.randint(0, (keep - sinks) // 2))
        c.pop("name", None)
        if _cost(c) <= top["window_prompt" if kind == "window_chunk" else kind]:
            return c


def _cost(case):
    """What the plain form's largest tensors hold, in elements."""
    H_q, H_kv, kind = case["H_q"], case["H_kv"], case["kind"]
    if kind == "window_prompt":
        tiles = -(-case["N"] // TILE)
        return case["B"] * tiles * TILE * _most_blocks(case, TILE, case["N"]) * TILE * (H_q + H_kv)
    if kind == "window_chunk":
        tiles = -(-case["N_q"] // TILE)
        return case["B"] * tiles * TILE * _most_blocks(case, TILE, case["len_hi"]) * TILE * (H_q + H_kv)
    if kind == "evict":
        return case["B"] * H_kv * D * (case["len_hi"] + case["keep"])
    n = _most_blocks(case, 1, case["len_hi"]) * TILE if kind == "window_decode" else case["len_hi"]
    return case["B"] * (H_kv * D + 4 * H_q) * n


def _most_blocks(case, rows, keys):
    return min(-(-keys // TILE), -(-case["sinks"] // TILE) + (case["window"] + rows - 2 + TILE) // TILE + 1)


def _lengths(case):
    """Context lengths of a batch: a function of the case, so that its work is."""
    r = random.Random("%d %d %d" % (case["B"], case["len_lo"], case["len_hi"]))
    return [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["B"])]


def _seen(p, window, sinks):
    """How many keys a query at position p sees."""
    first = max(0, p - window + 1)
    return p + 1 - first + min(sinks, first)


def work(case):
    H_q, H_kv, kind = case["H_q"], case["H_kv"], case["kind"]
    cached = H_kv * (64 + 8 + D) + 2 * H_q   # bytes of one token in the cache
    per_query = H_q * (64 + 8 + 2 * D)       # its codes and scales, its output
    if kind == "window_prompt":
        pairs = case["B"] * sum(_seen(p, case["window"], case["sinks"]) for p in range(case["N"]))
        return {"bytes": case["B"] * case["N"] * (cached + per_query), "flops": 4 * D * H_q * pairs}
    lens = _lengths(case)
    if kind == "window_chunk":
        n, w, s = case["N_q"], case["window"], case["sinks"]
        pairs = sum(_seen(L - n + i, w, s) for L in lens for i in range(n))
        read = sum(min(L, n + w - 1 + s) for L in lens)
        return {"bytes": read * cached + len(lens) * n * per_query, "flops": 4 * D * H_q * pairs}
    if kind == "window_decode":
        seen = sum(_seen(L - 1, case["window"], case["sinks"]) for L in lens)
        return {"bytes": seen * cached + len(lens) * per_query, "flops": 4 * D * H_q * seen}
    if kind == "weights_decode":
        return {"bytes": sum(lens) * (cached + 8 * H_kv) + len(lens) * per_query, "flops": 4 * D * H_q * sum(lens)}
    kept = sum(min(L, case["keep"]) for L in lens)
    return {"bytes": sum(lens) * 4 * H_kv + kept * (2 * cached + 8 * H_kv), "flops": 0}


# ---------------------------------------------------------------------------------------------------- inputs
def _aligned(t):
    """The tensor's bytes at an address that is a multiple of 1024, as the library asks for its tiles."""
    t = t.contiguous()
    n = t.numel() * t.element_size()
    raw = torch.empty(n + 1024, dtype=torch.uint8, device=t.device)
    at = -raw.data_ptr() % 1024
    out = raw[at:at + n].view(t.dtype).view(t.shape)
    out.copy_(t)
    return out


def _nvfp4(x, d):
    """x [..., 128] in units of d (broadcastable to [..., 1]): codes [..., 64] and scales [..., 8], both uint8."""
    y = (x / d).unflatten(-1, (8, 16))
    s = (y.abs().amax(-1, keepdim=True) / 6).clamp(max=448.0).to(torch.float8_e4m3fn)
    f = s.float()
    y = torch.where(f > 0, y / f, torch.zeros_like(y))
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    c = (torch.bucketize(y.abs(), edges) + (y < 0) * 8).to(torch.uint8).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), s.squeeze(-1).view(torch.uint8)


def _tiles(codes, sf):
    """codes [B,H,N,64], scales [B,H,N,8] -> the tile layout: codes [B,H,N_pad,64], sf [B,H,N_pad/128,2,512]."""
    B, H, N, _ = codes.shape
    pad = (0, 0, 0, -N % TILE)
    codes, sf = torch.nn.functional.pad(codes, pad), torch.nn.functional.pad(sf, pad)
    sf = sf.view(B, H, -1, 4, 32, 2, 4).permute(0, 1, 2, 5, 4, 3, 6).reshape(B, H, -1, 2, 512)
    return _aligned(codes), _aligned(sf)


def _swap(x, groups, by):
    """Groups `groups` of the last axis of x [..., rows, n] change places: group c of a row goes to c ^ by[row]."""
    y = x.unflatten(-1, (groups, -1))
    at = (torch.arange(groups, device=x.device) ^ by[:, None])
    return torch.take_along_dim(y, at.view(*([1] * (y.dim() - 3)), *at.shape, 1), -2).flatten(-2)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _stats(g, B, H_q, H_kv):
    """Means and tensor scales of B requests: the means' size is that of the offsets that models have."""
    amax = torch.rand(2, B, generator=g, device="cuda") * 0.5 + 1.0
    return {"q_mean": _normal(g, B, H_q, D), "k_mean": _normal(g, B, H_kv, D), "q_gscale": 5.5 * amax[0] / 2688.0,
            "k_gscale": 40.0 * amax[1] / 2688.0}


def _keys(g, factor, *shape):
    return _normal(g, *shape, D) * factor


def _outliers(g, H_kv):
    f = torch.ones(H_kv * D, device="cuda")
    f[torch.randperm(H_kv * D, generator=g, device="cuda")[:max(1, H_kv * D // 100)]] = 8.0
    return f.view(H_kv, D)


def _pages(g, case, lens, visible, extra=0):
    """A paged cache whose requests have `lens` tokens; visible(b, page): whether the page exists.  extra: more pages, empty ones."""
    H_q, H_kv, B = case["H_q"], case["H_kv"], len(lens)
    rows = [[i for i in range(-(-L // PAGE)) if visible(b, i)] for b, L in enumerate(lens)]
    n = sum(len(r) for r in rows)
    order = torch.randperm(n + extra + 1, generator=g, device="cuda")
    owner = torch.tensor([b for b, r in enumerate(rows) for _ in r], device="cuda")
    index = torch.tensor([i for r in rows for i in r], device="cuda")
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table = torch.full((B, max(-(-L // PAGE) for L in lens)), -1, dtype=torch.int32, device="cuda")
    table[owner, index] = order[:n].to(torch.int32)
    st = _stats(g, B, H_q, H_kv)
    live = (index * PAGE)[:, None] + torch.arange(PAGE, device="cuda") < lens_t[owner][:, None]   # [n, 64]
    kc = torch.zeros(n + extra + 1, H_kv, 4096, dtype=torch.uint8, device="cuda")
    ks = torch.zeros(n + extra + 1, H_kv, 512, dtype=torch.uint8, device="cuda")
    v8 = torch.zeros(n + extra + 1, H_kv, 8192, dtype=torch.uint8, device="cuda")
    dl = torch.zeros(n + extra + 1, H_q, PAGE, dtype=torch.bfloat16, device="cuda")
    t8 = torch.arange(PAGE, device="cuda") % 8
    factor, group = _outliers(g, H_kv)[:, None], torch.arange(H_q, device="cuda") % (H_q // H_kv)
    step = max(1, (1 << 27) // (H_kv * PAGE * D))
    for at in range(0, n, step):
        to, b, ok = order[at:min(n, at + step)], owner[at:at + step], live[at:at + step]
        k = _keys(g, factor, to.numel(), H_kv, PAGE) * ok[:, None, :, None]
        codes, sf = _nvfp4(k, st["k_gscale"][b].view(-1, 1, 1, 1))
        q_mean = st["q_mean"].view(B, H_kv, -1, D)[b] / (st["q_gscale"] * st["k_gscale"])[b].view(-1, 1, 1, 1)
        delta = (q_mean @ k.mT).flatten(1, 2)                        # [pages, H_q, 64]
        v = (_normal(g, to.numel(), H_kv, PAGE, D) * ok[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        kc[to], ks[to] = _swap(codes, 4, t8 // 2).flatten(2), sf.flatten(2)
        v8[to], dl[to] = _swap(v, 8, t8).flatten(2), _swap(delta, 8, group).bfloat16()
    return {"k_codes": kc, "k_sf": ks, "v_fp8": v8, "delta": dl, "table": table, "lens": lens_t, "lens_host": lens, "stats": st,
            "spare": order[n:n + extra].to(torch.int32)}


def _query(g, st, *shape):
    """Centered queries, quantized: [B, H_q, N, 128] in the tile layout."""
    return _tiles(*_nvfp4(_normal(g, *shape, D), st["q_gscale"].view(-1, 1, 1, 1)))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind, B, H_q, H_kv = case["kind"], case["B"], case["H_q"], case["H_kv"]
    st = {"case": dict(case), "scale": 1.0 / math.sqrt(D), "v_scale": 0.5, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if kind == "window_prompt":
        N = case["N"]
        x = _stats(g, B, H_q, H_kv)
        k = _keys(g, _outliers(g, H_kv)[:, None], B, H_kv, N)
        q_mean = x["q_mean"].view(B, H_kv, -1, D) / (x["q_gscale"] * x["k_gscale"]).view(-1, 1, 1, 1)
        delta = torch.nn.functional.pad((q_mean @ k.mT).flatten(1, 2), (0, -N % TILE)).bfloat16()
        v = torch.nn.functional.pad(_normal(g, B, H_kv, N, D), (0, 0, 0, -N % TILE)).to(torch.float8_e4m3fn).view(torch.uint8)
        st.update(stats=x, q=_query(g, x, B, H_q, N), k=_tiles(*_nvfp4(k, x["k_gscale"].view(-1, 1, 1, 1))), v_fp8=_aligned(v),
                  delta=_aligned(delta), out=torch.empty(B, N, H_q, D, dtype=torch.bfloat16, device="cuda"))
        return st
    lens = _lengths(case)
    if kind == "evict":
        keep = case["keep"]
        per = -(-keep // PAGE)
        st.update(_pages(g, case, lens, lambda b, i: True, extra=B * per))
        slots = st["table"].shape[1] * PAGE
        # what a few hundred steps leave behind: most tokens little, some much, the newest not much yet
        age = (st["lens"].view(B, 1, 1) - torch.arange(slots, device="cuda")).clamp(min=0)
        heavy = torch.exp(1.5 * _normal(g, B, H_kv, slots))
        st.update(weights=heavy * (age / 512.0).clamp(max=1.0), new_table=st["spare"].view(B, per),
                  kept=torch.empty(B, H_kv, keep, dtype=torch.int32, device="cuda"), new_lens=torch.empty_like(st["lens"]),
                  new_weights=torch.empty(B, H_kv, max(slots, per * PAGE), device="cuda"))
        return st
    w, s = case["window"], case["sinks"]
    n = case.get("N_q", 1)
    if kind == "weights_decode":
        st.update(_pages(g, case, lens, lambda b, i: True))
        slots = st["table"].shape[1] * PAGE
        # sums of some 64 steps: their mean is 64 steps' worth of a key's share, most keys have less and some much more
        L = st["lens"].view(B, 1, 1)
        held = torch.exp(1.5 * _normal(g, B, H_kv, slots)) * (64 * H_q / H_kv / L) * (torch.arange(slots, device="cuda") < L - 1)
        st.update(weights=held)
    else:
        st.update(_pages(g, case, lens, lambda b, i: i * PAGE < s or (i + 1) * PAGE > lens[b] - n - w + 1))
    st.update(q=_query(g, st["stats"], B, H_q, n), out=torch.empty(B, n, H_q, D, dtype=torch.bfloat16, device="cuda"))
    if kind != "window_chunk":
        st["out"] = st["out"].view(B, H_q, D)
        # more than the partition states of any batch here, as a server would set aside once
        parts = -(-st["table"].shape[1] // (PART * 2))
        room = B * H_q * (parts * (D + 2) + 66) * 4 + (B * H_q * st["table"].shape[1] * PAGE * 4 if kind == "weights_decode" else 0)
        st["workspace"] = torch.empty(room + 4096, dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------- the plain forms
def _values(device):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=device)


def _decoded(codes, sf):
    """codes [..., 64], scales [..., 8] -> [..., 128] in units of the tensor scale."""
    x = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return _values(codes.device)[x.int()] * sf.view(torch.float8_e4m3fn).float().repeat_interleave(16, -1)


def _untiled(codes, sf):
    B, H, n, _ = codes.shape
    return _decoded(codes, sf.view(B, H, -1, 2, 32, 4, 4).permute(0, 1, 2, 5, 4, 3, 6).reshape(B, H, n, 8))


def _attend(S, V, lam, v_scale, part):
    """S [..., blocks, G, rows, 128] masked logits, V [..., blocks, 128 keys, 128]; blocks ascending, visited from the last to the first;
    the running maximum starts anew every `part` blocks from the first (0: never).  -> out [..., G, rows, 128], m, l."""
    n = S.shape[-4]
    block = S.amax(-1, keepdim=True)                                     # [..., blocks, G, rows, 1]
    parts = block.unflatten(-4, (-1, part)) if part else block.unsqueeze(-5)
    m = parts.flip(-4).cummax(-4).values.flip(-4).flatten(-5, -4)
    top = block.amax(-4, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    safe = torch.where(m == -math.inf, top, m)
    P = torch.exp2((S - safe) * lam)
    w = torch.exp2((m - top) * lam)                                       # 0 where nothing is visible yet
    l = (w * P.sum(-1, keepdim=True)).sum(-4)
    P = (448.0 * P).to(torch.float8_e4m3fn).float()
    rows = P.flatten(-3, -2) @ V                                          # [..., blocks, G rows, 128]
    O = (w * rows.unflatten(-2, P.shape[-3:-1])).sum(-4)
    out = torch.where(l > 0, O / (448.0 * l.clamp(min=1e-30)) * v_scale, torch.zeros_like(O))
    return out, top.squeeze(-4), l


def _lam(st):
    x = st["stats"]
    return (st["scale"] * LOG2E) * x["q_gscale"] * x["k_gscale"]


def _block_lists(first, last, window, sinks, n):
    """Blocks that hold a key visible to some query at positions first..last (tensors [...]): [..., n] ascending, -1 where there is none."""
    low = (first - window + 1).clamp(min=0) // TILE
    k = torch.arange(n, device=first.device)
    heads = torch.minimum(torch.full_like(low, -(-sinks // TILE)), low)[..., None]
    at = torch.where(k < heads, k, k - heads + low[..., None])
    return torch.where((at <= last[..., None] // TILE) & (last[..., None] >= 0), at, -1)


def _mask(keys, pos, window, sinks):
    """keys [..., blocks, 128], pos [..., rows] -> [..., blocks, rows, 128]"""
    j, p = keys[..., :, None, :], pos[..., None, :, None]
    return (j >= 0) & (j <= p) & ((j > p - window) | (j < sinks))


def _page_gather(st, blocks):
    """K [B, ..., H_kv, 128, 128], V, Delta_S [B, ..., H_q, 128] of the blocks [B, ...] (those that do not exist: some page)."""
    H_kv, H_q = st["k_codes"].shape[1], st["delta"].shape[1]
    B, table = blocks.shape[0], st["table"]
    index = (blocks.clamp(min=0)[..., None] * 2 + torch.arange(2, device=blocks.device)).clamp(max=table.shape[1] - 1)
    pages = table[torch.arange(B, device=blocks.device).view(-1, *([1] * (index.dim() - 1))), index].clamp(min=0).long()
    t8 = torch.arange(PAGE, device=blocks.device) % 8
    kc = _swap(st["k_codes"][pages].unflatten(-1, (PAGE, 64)), 4, t8 // 2)        # [B, ..., 2, H_kv, 64, 64]
    K = _decoded(kc, st["k_sf"][pages].unflatten(-1, (PAGE, 8)))
    V = _swap(st["v_fp8"][pages].unflatten(-1, (PAGE, D)), 8, t8).view(torch.float8_e4m3fn).float()
    dl = _swap(st["delta"][pages], 8, torch.arange(H_q, device=blocks.device) % (H_q // H_kv)).float()   # [B, ..., 2, H_q, 64]
    return K.transpose(-4, -3).flatten(-3, -2), V.transpose(-4, -3).flatten(-3, -2), dl.transpose(-3, -2).flatten(-2)


def _plain_rows(st, q, blocks, pos, K, V, dl, lens):
    """q [B,H_q,tiles,128,128], blocks [B,tiles,n], pos [B,tiles,128], K, V [B,tiles,n,H_kv,128,128], dl [B,tiles,n,H_q,128]
    -> [B,H_q,tiles,128,128]"""
    case = st["case"]
    G = case["H_q"] // case["H_kv"]
    keys = torch.where(blocks[..., None] >= 0, blocks[..., None] * TILE + torch.arange(TILE, device=blocks.device), -1)
    seen = _mask(torch.where(keys < lens.view(-1, 1, 1, 1), keys, -1), pos, case["window"], case["sinks"])      # [B,tiles,n,rows,128]
    q = q.unflatten(1, (-1, G)).permute(0, 3, 1, 2, 4, 5).flatten(3, 4)                 # [B,tiles,H_kv,G*128,128]
    S = q[:, :, :, None] @ K.permute(0, 1, 3, 2, 5, 4)                                 # [B,tiles,H_kv,n,G*128,128]
    S = S.unflatten(-2, (G, -1)) + dl.unflatten(3, (-1, G)).permute(0, 1, 3, 2, 4, 5)[..., None, :]
    S = S.masked_fill_(~seen[:, :, None, :, None], -math.inf)
    out, _, _ = _attend(S, V.transpose(2, 3), _lam(st).view(-1, 1, 1, 1, 1, 1, 1), st["v_scale"], 0)
    return out.permute(0, 2, 3, 1, 4, 5).flatten(1, 2)


def _plain_prompt(st):
    case = st["case"]
    B, N, H_q, H_kv = case["B"], case["N"], case["H_q"], case["H_kv"]
    q, k = _untiled(*st["q"]).unflatten(2, (-1, TILE)), _untiled(*st["k"]).unflatten(2, (-1, TILE))
    v = st["v_fp8"].view(torch.float8_e4m3fn).float().unflatten(2, (-1, TILE))
    first = torch.arange(q.shape[2], device=q.device) * TILE
    blocks = _block_lists(first, (first + TILE - 1).clamp(max=N - 1), case["window"], case["sinks"], _most_blocks(case, TILE, N))
    at = blocks.clamp(min=0)
    pos = (first[:, None] + torch.arange(TILE, device=q.device)).clamp(max=N - 1)
    out = _plain_rows(st, q, blocks.expand(B, -1, -1), pos.expand(B, -1, -1), k[:, :, at].permute(0, 2, 3, 1, 4, 5),
                      v[:, :, at].permute(0, 2, 3, 1, 4, 5), st["delta"].float().unflatten(2, (-1, TILE))[:, :, at].permute(0, 2, 3, 1, 4),
                      torch.full((B,), N, device=q.device))
    return out.flatten(2, 3)[:, :, :N].transpose(1, 2).bfloat16()


def _plain_chunk(st):
    case = st["case"]
    N_q, lens = case["N_q"], st["lens"].long()
    q = _untiled(*st["q"]).unflatten(2, (-1, TILE))
    row0 = torch.arange(q.shape[2], device=q.device) * TILE
    shift = (lens - N_q)[:, None]
    blocks = _block_lists(row0 + shift, (row0 + TILE - 1).clamp(max=N_q - 1) + shift, case["window"], case["sinks"],
                          _most_blocks(case, TILE, case["len_hi"]))
    pos = (row0[:, None] + torch.arange(TILE, device=q.device)).clamp(max=N_q - 1) + shift[..., None]
    out = _plain_rows(st, q, blocks, pos, *_page_gather(st, blocks), lens)
    return out.flatten(2, 3)[:, :, :N_q].transpose(1, 2).bfloat16()


def _plain_decode(st, blocks, window, sinks):
    """blocks [B, n] ascending, -1 at the end -> out [B, H_q, 128], S [B, H_kv, n, G, 1, 128], m, l"""
    case, lens = st["case"], st["lens"].long()
    G = case["H_q"] // case["H_kv"]
    blocks = torch.nn.functional.pad(blocks, (0, -blocks.shape[1] % PART), value=-1)
    K, V, dl = _page_gather(st, blocks)                                               # [B, n, H_kv, 128, 128], [B, n, H_q, 128]
    keys = torch.where(blocks[..., None] >= 0, blocks[..., None] * TILE + torch.arange(TILE, device=blocks.device), -1)
    seen = _mask(keys, lens[:, None] - 1, window, sinks)                              # [B, n, 1, 128]
    q = _untiled(*st["q"])[:, :, :1].unflatten(1, (-1, G)).squeeze(3)                 # [B, H_kv, G, 128]
    S = q[:, None] @ K.mT + dl.unflatten(2, (-1, G))                                  # [B, n, H_kv, G, 128]
    S = S.transpose(1, 2)[..., None, :].masked_fill(~seen[:, None, :, None], -math.inf)
    lam = _lam(st).view(-1, 1, 1, 1, 1, 1)
    out, m, l = _attend(S, V.transpose(1, 2), lam, st["v_scale"], PART)
    return out.flatten(1, 3).bfloat16(), S, m, l


def _plain_window_decode(st):
    case = st["case"]
    last = st["lens"].long() - 1
    return _plain_decode(st, _block_lists(last, last, case["window"], case["sinks"], _most_blocks(case, 1, case["len_hi"])),
                         case["window"], case["sinks"])[0]


def _plain_weights(st):
    last = st["lens"].long() - 1
    far = st["table"].shape[1] * PAGE
    blocks = _block_lists(last, last, far, 0, -(-far // TILE))
    out, S, m, l = _plain_decode(st, blocks, far, 0)
    P = torch.exp2((S - m.unsqueeze(2)) * _lam(st).view(-1, 1, 1, 1, 1, 1)) / l.unsqueeze(2)
    st["weights"] += P.sum(3).flatten(2)[..., :far]
    st["out"].copy_(out)
    return [st["out"], st["weights"]]


def _plain_evict(st):
    case, lens = st["case"], st["lens"].long()
    keep, sinks, recent = case["keep"], case["sinks"], case["recent"]
    B, H_kv, slots = st["weights"].shape
    L, at = lens.view(-1, 1, 1), torch.arange(slots, device="cuda")
    # two stable sorts, the second the weightier: protected tokens first, then by weight, equal ones by slot, what does not exist last
    rank = torch.where(at >= L, 2, torch.where((at < sinks) | (at >= L - recent), 0, 1)).expand(B, H_kv, slots)
    order = st["weights"].sort(dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, rank.gather(-1, order).sort(dim=-1, stable=True).indices)[..., :keep]
    kept = torch.where(torch.arange(order.shape[-1], device="cuda") < L, order, slots).sort(-1).values
    kept = torch.nn.functional.pad(torch.where(kept < slots, kept, -1), (0, keep - kept.shape[-1]), value=-1)
    n = lens.clamp(max=keep)
    have = kept >= 0
    src = kept.clamp(min=0)
    st["kept"].copy_(kept)
    st["new_lens"].copy_(n)
    st["new_weights"].zero_()[..., :keep].copy_(st["weights"].gather(-1, src) * have)
    # the tokens, page by page: gathered from their slots, zeros past the end
    per = st["new_table"].shape[1]
    fill = (0, per * PAGE - keep)
    src, have = torch.nn.functional.pad(src, fill), torch.nn.functional.pad(have, fill)
    H_q, G = case["H_q"], case["H_q"] // H_kv
    page, slot = st["table"].gather(1, (src // PAGE).flatten(1)).view_as(src).long(), src % PAGE
    hk, t8 = torch.arange(H_kv, device="cuda").view(1, -1, 1), torch.arange(PAGE, device="cuda") % 8
    dst = st["new_table"].long()
    ok = have.unflatten(-1, (per, PAGE)).transpose(1, 2)                               # [B, pages, H_kv, 64]
    for name, width, groups, by in (("k_codes", 64, 4, slot % 8 // 2), ("v_fp8", D, 8, slot % 8), ("k_sf", 8, 1, slot * 0)):
        pool = st[name].unflatten(-1, (PAGE, width))
        rows = pool[page, hk, slot].unflatten(-1, (groups, -1))                         # [B, H_kv, keep, groups, bytes]
        rows = torch.take_along_dim(rows, (torch.arange(groups, device="cuda") ^ by[..., None])[..., None], -2).flatten(-2)
        rows = rows.unflatten(2, (per, PAGE)).transpose(1, 2) * ok[..., None]
        st[name][dst] = _swap(rows, groups, {4: t8 // 2, 8: t8, 1: t8 * 0}[groups]).flatten(3)
    hq = torch.arange(H_q, device="cuda")
    page, slot, ok = (x.repeat_interleave(G, 1 if x is not ok else 2) for x in (page, slot, ok))
    dl = st["delta"][page, hq.view(1, -1, 1), ((slot // 8) ^ (hq % G).view(1, -1, 1)) * 8 + slot % 8]
    dl = torch.where(ok, dl.unflatten(2, (per, PAGE)).transpose(1, 2), torch.zeros((), dtype=dl.dtype, device="cuda"))
    st["delta"][dst] = _swap(dl, 8, hq % G)
    return _evicted(st)


def _evicted(st):
    """The pools whole, codes as bytes: the operator moves them and computes none."""
    return [st["kept"], st["new_lens"], st["new_weights"], st["k_codes"], st["k_sf"], st["v_fp8"], st["delta"]]


# ---------------------------------------------------------------------------------------------------- a pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own(st, kind)
    if kind == "window_prompt":
        return _plain_prompt(st)
    if kind == "window_chunk":
        return _plain_chunk(st)
    if kind == "window_decode":
        return _plain_window_decode(st)
    if kind == "weights_decode":
        return _plain_weights(st)
    return _plain_evict(st)


def _own(st, kind):
    from paper_2609_33135_b200 import binding
    case = st["case"]
    H_q, H_kv = case["H_q"], case["H_kv"]
    stats = binding.Stats(**st["stats"])
    if kind == "window_prompt":
        q, k = binding.Fp4Tensor(*st["q"], case["B"], H_q, case["N"]), binding.Fp4Tensor(*st["k"], case["B"], H_kv, case["N"])
        binding.mpfa_prefill_window(q, k, st["v_fp8"], st["delta"], stats, st["v_scale"], case["window"], case["sinks"], st["scale"],
                                    st["out"], None, st["status"])
        return st["out"]
    kv = binding.PagedKV(st["k_codes"], st["k_sf"], st["v_fp8"], st["delta"], st["k_codes"].shape[0], H_q, H_kv)
    if kind == "evict":
        binding.mpfa_evict_paged(kv, st["table"], st["lens"], st["weights"], case["keep"], case["sinks"], case["recent"],
                                 st["new_table"], st["kept"], st["new_lens"], st["new_weights"], st["status"])
        return _evicted(st)
    q = binding.Fp4Tensor(*st["q"], case["B"], H_q, case.get("N_q", 1))
    if kind == "window_chunk":
        binding.mpfa_prefill_paged_window(q, kv, st["table"], st["lens"], stats, st["v_scale"], case["window"], case["sinks"],
                                          st["scale"], st["out"], None, st["status"])
        return st["out"]
    if kind == "window_decode":
        binding.mpfa_decode_window(q, kv, st["table"], st["lens"], stats, st["v_scale"], case["window"], case["sinks"], st["scale"],
                                   st["out"], None, st["workspace"], st["status"])
        return st["out"]
    binding.mpfa_decode_weights(q, kv, st["table"], st["lens"], stats, st["v_scale"], st["scale"], st["weights"], st["out"], None,
                                st["workspace"], st["status"])
    return [st["out"], st["weights"]]


# ---------------------------------------------------------------------------------------------------- in 64 bits, from the definition
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "evict":
        return _exact_evict(st)
    if case["kind"] == "window_prompt":
        return _exact_prompt(st)
    return _exact_paged(st)


def _e2m1(nibble):
    """(-1)^s 2^(e-1) (1 + m/2), e = 0: m/2"""
    n = nibble.long()
    e, m = (n >> 1) & 3, (n & 1).double()
    mag = torch.where(e == 0, 0.5 * m, torch.exp2(e.double() - 1) * (1 + 0.5 * m))
    return torch.where(n >= 8, -mag, mag)


def _e4m3(byte):
    n = byte.long()
    e, m = (n >> 3) & 15, (n & 7).double()
    mag = torch.where(e == 0, m * 2.0 ** -9, torch.exp2(e.double() - 7) * (1 + m / 8))
    return torch.where(n >= 128, -mag, mag)


def _p_hat(x):
    """x in [0, 448] to the nearest E4M3 value, ties to the even one"""
    step = torch.exp2(torch.floor(torch.log2(x.clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _rows64(S, V, lam, v_scale, groups):
    """S [rows, keys] with -inf where hidden; groups: lists of slices of the key axis, each visited last to first with a maximum of its own."""
    top = S.amax(1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    O, l = torch.zeros(S.shape[0], D, dtype=torch.float64, device=S.device), torch.zeros(S.shape[0], 1, dtype=torch.float64, device=S.device)
    for slices in groups:
        m = torch.full_like(top, -math.inf)
        for at in reversed(slices):
            m = torch.maximum(m, S[:, at].amax(1, keepdim=True))
            P = torch.exp2(lam * (S[:, at] - torch.where(torch.isinf(m), top, m)))
            w = torch.exp2(lam * (m - top))
            l += w * P.sum(1, keepdim=True)
            O += w * (_p_hat(448.0 * P) @ V[at])
    return torch.where(l > 0, O / (448.0 * l) * v_scale, torch.zeros_like(O)), top, l


def _exact_lam(st, b):
    return st["scale"] / math.log(2.0) * float(st["stats"]["q_gscale"][b]) * float(st["stats"]["k_gscale"][b])


def _tile_rows(codes, sf, b, h, n):
    """n rows of head h from the tile layout, by its index map"""
    t, g = torch.arange(n, device=codes.device)[:, None], torch.arange(8, device=codes.device)
    scale = _e4m3(sf[b, h].flatten()[t // 128 * 1024 + g // 4 * 512 + t % 32 * 16 + t % 128 // 32 * 4 + g % 4])
    c = codes[b, h, :n]
    x = torch.zeros(n, D, dtype=torch.float64, device=codes.device)
    x[:, 0::2], x[:, 1::2] = _e2m1(c & 15), _e2m1(c >> 4)
    return (x.view(n, 8, 16) * scale[:, :, None]).view(n, D)


def _exact_prompt(st):
    case = st["case"]
    B, N, H_q, H_kv, w, s = (case[k] for k in ("B", "N", "H_q", "H_kv", "window", "sinks"))
    out = torch.zeros(B, N, H_q, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        lam = _exact_lam(st, b)
        for hk in range(H_kv):
            K, V = _tile_rows(*st["k"], b, hk, N), _e4m3(st["v_fp8"][b, hk, :N])
            for h in range(hk * (H_q // H_kv), (hk + 1) * (H_q // H_kv)):
                q, delta = _tile_rows(*st["q"], b, h, N), st["delta"][b, h, :N].double()
                for r in range(0, N, 1024):
                    i = torch.arange(r, min(N, r + 1024), device="cuda")
                    low = max(0, r - w + 1) // 128 * 128
                    head = min(low, -(-s // 128) * 128)          # keys [0, head) and [low, end) hold all that these rows see
                    j = torch.cat((torch.arange(head, device="cuda"), torch.arange(low, int(i[-1]) + 1, device="cuda")))
                    S = q[i] @ K[j].T + delta[j]
                    S[~((j <= i[:, None]) & ((j > i[:, None] - w) | (j < s)))] = -math.inf
                    O, _, _ = _rows64(S, V[j], lam, st["v_scale"], [[slice(a, a + 128) for a in range(0, j.numel(), 128)]])
                    out[b, i, h] = O
    return out


def _exact_paged(st):
    case = st["case"]
    kind, B, H_q, H_kv = case["kind"], case["B"], case["H_q"], case["H_kv"]
    n, G = case.get("N_q", 1), H_q // H_kv
    out = torch.zeros(B, n, H_q, D, dtype=torch.float64, device="cuda")
    weights = st["weights"].double() if kind == "weights_decode" else None
    t, g, byte = torch.arange(PAGE)[:, None], torch.arange(64)[None] // 8, torch.arange(64)[None] % 8
    at_k = (t // 8 * 512 + t % 8 * 64 + ((g // 2) ^ (t % 8 // 2)) * 16 + g % 2 * 8 + byte).cuda()
    c = torch.arange(D)[None]
    at_v = (t // 8 * 1024 + t % 8 * 128 + ((c // 16) ^ (t % 8)) * 16 + c % 16).cuda()
    for b, L in enumerate(st["lens_host"]):
        w, s = (case["window"], case["sinks"]) if kind != "weights_decode" else (L, 0)
        lam = _exact_lam(st, b)
        low = max(0, L - n - w + 1) // 128 * 128
        j = torch.arange(L, device="cuda")
        j = j[(j >= low) | (j < -(-s // 128) * 128)]
        pages, where = torch.unique(j // PAGE, return_inverse=True)
        ids = st["table"][b, pages].long().clamp(min=0)
        where = where * PAGE + j % PAGE
        i = torch.arange(L - n, L, device="cuda")[:, None]
        hidden = ~((j <= i) & ((j > i - w) | (j < s)))
        if kind == "window_chunk":   # a row visits only its own tile's blocks: the others hold nothing it sees
            groups = [[slice(a, a + 128) for a in range(0, j.numel(), 128)]]
        else:
            groups = [[slice(a, min(a + 128, j.numel())) for a in range(p, min(p + 1024, j.numel()), 128)] for p in range(0, j.numel(), 1024)]
        for hk in range(H_kv):
            kc = st["k_codes"][ids, hk][:, at_k].flatten(0, 1)[where]
            K = torch.stack((_e2m1(kc & 15), _e2m1(kc >> 4)), -1).flatten(1)
            K = (K.view(-1, 8, 16) * _e4m3(st["k_sf"][ids, hk].view(-1, 8)[where])[:, :, None]).view(-1, D)
            V = _e4m3(st["v_fp8"][ids, hk][:, at_v].flatten(0, 1)[where])
            for h in range(hk * G, hk * G + G):
                tt = torch.arange(PAGE, device="cuda")
                delta = st["delta"][ids, h][:, ((tt // 8) ^ (h % G)) * 8 + tt % 8].flatten()[where].double()
                S = _tile_rows(*st["q"], b, h, n) @ K.T + delta
                S[hidden] = -math.inf
                O, top, l = _rows64(S, V, lam, st["v_scale"], groups)
                out[b, :, h] = O
                if weights is not None:
                    weights[b, hk, :L] += torch.exp2(lam * (S[0] - top[0])) / l[0]
    if kind == "window_chunk":
        return out
    out = out.view(B, H_q, D)
    return out if weights is None else [out, weights]


def _exact_evict(st):
    case = st["case"]
    keep, sinks, recent = case["keep"], case["sinks"], case["recent"]
    w = st["weights"].cpu().double()
    B, H_kv, slots = w.shape
    kept = torch.full((B, H_kv, keep), -1, dtype=torch.int32)
    out = torch.zeros(st["new_weights"].shape, dtype=torch.float64)
    lens = st["lens_host"]
    for b, L in enumerate(lens):
        for hk in range(H_kv):
            slot = list(range(L))
            if L > keep:
                x = w[b, hk].tolist()
                middle = sorted(range(sinks, L - recent), key=lambda j: (-x[j], j))[:keep - sinks - recent]
                slot = list(range(sinks)) + sorted(middle) + list(range(L - recent, L))
            kept[b, hk, :len(slot)] = torch.tensor(slot, dtype=torch.int32)
            out[b, hk, :len(slot)] = w[b, hk, slot]
    return [kept, torch.tensor([min(L, keep) for L in lens], dtype=torch.int32), out, None, None, None, None]
