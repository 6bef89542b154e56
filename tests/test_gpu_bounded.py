"""GPU: attention with a sliding window and sinks (prefill, chunks on pages, decode), decode that sums attention weights, and eviction,
against the 64-bit statements of bounded_plain.py."""
import contextlib
import os

import numpy as np
import pytest
import torch

import bounded_plain as plain
from paper_2609_33135_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def binding():
    from paper_2609_33135_b200 import binding as B
    return B


@contextlib.contextmanager
def arrangement(a):
    """The prefill calls' work arrangement; afterwards the one that the suite runs with."""
    binding().mpfa_set_prefill_arrangement(a)
    try:
        yield
    finally:
        binding().mpfa_set_prefill_arrangement(int(os.environ.get("MPFA_TEST_ARRANGEMENT", "0")))


def state(seed, lens, H_q, H_kv, v_scale=1.0, smooth=True):
    from paper_2609_33135_b200 import decode_cache
    w = wl.decode_workload("bounded", seed, len(lens), H_q, H_kv, 1, max(max(lens), 1), seq_lens=[max(L, 1) for L in lens])
    st = decode_cache.build_cache(w, v_scale=v_scale, smooth=smooth)
    st.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return st


def close(got, want, room, what):
    d = np.abs(got.astype(np.float64) - want)
    assert np.isfinite(got).all(), what
    worst = np.unravel_index(np.argmax(d - room), d.shape)
    assert (d <= room).all(), (what, worst, float(got[worst]), float(want[worst]), float(room[worst]))


def rounded(out, out_f32):
    assert torch.equal(out, out_f32.to(torch.bfloat16))


def window_decode(st, window, sinks, table=None, out_f32=True):
    B = binding()
    table = st.page_table if table is None else table
    out, o32 = torch.empty_like(st.out), torch.empty_like(st.out_f32)
    ws = B.decode_window_workspace(table.shape[0], st.kv.H_q, st.kv.H_kv, table.shape[1], window, sinks)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_decode_window(st.q4, st.kv, table, st.seq_lens, st.stats, st.v_scale, window, sinks, st.softmax_scale, out,
                         o32 if out_f32 else None, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    return out, o32


def check_window_decode(st, window, sinks, o32, requests=None):
    q = plain.tile_rows(st.q4)
    G = st.kv.H_q // st.kv.H_kv
    got = o32.cpu().numpy()
    for b in range(st.q4.B) if requests is None else requests:
        L = int(st.seq_lens[b])
        if L == 0:
            assert not got[b].any()
            continue
        K, V, D = plain.cached(st.kv, st.page_table[b].cpu().numpy(), L)
        see, lam = plain.visible([L - 1], L, window, sinks), plain.lam_of(st.stats, b, st.softmax_scale)
        for h in range(st.kv.H_q):
            want, room, _, _ = plain.attend(q[b, h], K[h // G], V[h // G], D[h], see, lam, st.v_scale, 8)
            close(got[b, h], want[0], room[0], (b, h, L, window, sinks))


@pytest.mark.parametrize("H_q,H_kv", [(4, 4), (4, 2), (6, 2), (8, 2), (10, 2), (12, 2), (14, 2), (16, 2)])
def test_window_decode_for_every_group(H_q, H_kv):
    st = state(900 + H_q, [1, 0, 64, 129, 1025, 2600], H_q, H_kv, v_scale=0.5)
    for window, sinks in ((1, 0), (130, 4), (1500, 300)):
        out, o32 = window_decode(st, window, sinks)
        rounded(out, o32)
        check_window_decode(st, window, sinks, o32)


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 127, 128, 129, 1000, 1024, 2303, 2304, 2305, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("sinks", [0, 1, 4, 63, 64, 65, 128, 200, 2304, (1 << 31) - 1])
def test_window_decode_edges(window, sinks):
    """Windows and sinks that end before, on and behind the borders of pages and blocks, that touch, overlap and cover everything."""
    st = edges()
    out, o32 = window_decode(st, window, sinks)
    rounded(out, o32)
    check_window_decode(st, window, sinks, o32)


_edges = []


def edges():
    if not _edges:
        _edges.append(state(950, [2304, 2305, 2367, 700, 5], 4, 2))
    return _edges[0]


def test_window_decode_of_the_whole_context_is_decode():
    from paper_2609_33135_b200 import decode_cache
    st = state(951, [3000, 1, 0, 1024], 8, 2)
    decode_cache.decode_step(st)
    for window, sinks in ((3000, 0), (1 << 30, 7), (1, 3000)):
        out, o32 = window_decode(st, window, sinks)
        assert torch.equal(out, st.out) and torch.equal(o32, st.out_f32)


def test_window_decode_looks_at_no_page_and_no_value_that_is_hidden():
    """Pages out of view are given away (their entries are anything), and hidden tokens of the pages that stay hold NaN everywhere."""
    st = state(952, [2000, 1500, 90], 8, 2)
    window, sinks = 300, 70
    clean, _ = window_decode(st, window, sinks)
    table = st.page_table.clone()
    for b, L in enumerate((2000, 1500, 90)):
        low = max(L - window, 0)
        for i in range(-(-L // 64)):
            page = int(st.page_table[b, i])
            hidden = [t for t in range(64) if sinks <= i * 64 + t < low]
            if len(hidden) == 64:
                table[b, i] = (-1, 10 ** 9, -(2 ** 31))[i % 3]
                for pool in (st.kv.k_codes, st.kv.k_sf, st.kv.v_fp8):
                    pool[page] = 0x7F
                continue
            for t in hidden:
                st.kv.v_fp8[page, :, t * 128:t * 128 + 128] = 0x7F
                st.kv.k_sf[page, :, t * 8:t * 8 + 8] = 0x7F
                for h in range(8):
                    st.kv.delta[page, h, ((t // 8) ^ (h % 4)) * 8 + t % 8] = float("nan")
    out, o32 = window_decode(st, window, sinks, table)
    assert torch.equal(out, clean) and bool(torch.isfinite(o32).all())


def test_window_decode_reports_a_missing_page():
    B = binding()
    st = state(953, [700, 700], 4, 2)
    table = st.page_table.clone()
    table[1, 10] = 10 ** 8
    ws = B.decode_window_workspace(2, 4, 2, table.shape[1], 128, 0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty_like(st.out)
    B.mpfa_decode_window(st.q4, st.kv, table, st.seq_lens, st.stats, 1.0, 128, 0, st.softmax_scale, out, None, ws, status)
    assert int(status) == B.MPFA_DEV_BAD_PAGE
    want, _ = window_decode(st, 128, 0)
    assert torch.equal(out[0], want[0])


def test_window_decode_of_many_requests():
    """More requests than the kernel holds lengths for, so that work items are found by another rule; and a length past the table."""
    lens = [1 + (37 * i) % 400 for i in range(790)]
    st = state(954, lens, 4, 2)
    _, o32 = window_decode(st, 100, 3)
    check_window_decode(st, 100, 3, o32, [0, 1, 5, 100, 767, 768, 789])
    few = state(955, [500, 640], 4, 2)
    full, _ = window_decode(few, 200, 5)
    few.seq_lens[1] = 10 ** 6   # treated as 640
    out, _ = window_decode(few, 200, 5)
    assert torch.equal(out, full)


# ------------------------------------------------------------------------------------------------------------------ prefill
def check_rows(q, K, V, D, o32, pos, window, sinks, lam, v_scale, heads, what):
    """q [H_q, N, 128], K, V [H_kv, n_kv, 128], o32 [N, H_q, 128]; every 128-row tile visits its own blocks."""
    G = heads[0] // heads[1]
    for h in range(heads[0]):
        for r in range(0, len(pos), 128):
            rows = slice(r, min(r + 128, len(pos)))
            see = plain.visible(pos[rows], K.shape[1], window, sinks)
            want, room, _, _ = plain.attend(q[h, rows], K[h // G], V[h // G], D[h], see, lam, v_scale, 0)
            close(o32[rows, h], want, room, (what, h, r))


@pytest.mark.parametrize("B_,N_q,N_kv,H_q,H_kv,window,sinks", [
    (1, 1, 1, 1, 1, 1, 0),
    (2, 300, 300, 4, 2, 1, 0),            # each row sees its own key only
    (1, 300, 300, 4, 2, 1, 5),
    (1, 513, 513, 2, 1, 64, 130),         # more sinks than a block
    (1, 700, 700, 8, 1, 129, 4),
    (2, 257, 900, 4, 4, 200, 1),          # more keys than queries: the window's edge at an odd place of every block
    (1, 129, 2000, 10, 2, 700, 300),
    (1, 400, 150, 4, 2, 60, 3),           # more queries than keys: the first rows see nothing
    (1, 1000, 1000, 2, 2, 5000, 0),
    (1, 1000, 1000, 2, 2, (1 << 31) - 1, (1 << 31) - 1),
    (1, 200, 5000, 2, 1, 4600, 100),      # 37 blocks: accumulated in runs
    (1, 128, 4400, 1, 1, 10, 4300),       # sinks up to the window
])
def test_prefill_window(B_, N_q, N_kv, H_q, H_kv, window, sinks):
    B = binding()
    w = wl.prefill_workload("pw", 960 + N_q, B_, N_kv, H_q, H_kv, True, q_bias=True)
    q = w.q[:, :N_q] if N_q <= N_kv else wl.prefill_workload("pw", 961, B_, N_q, H_q, H_kv, True, q_bias=True).q
    s1 = B.stage1(q.contiguous().cuda(), w.k.cuda(), w.v.cuda(), v_scale=0.5)
    out = torch.empty(B_, N_q, H_q, 128, dtype=torch.bfloat16, device="cuda")
    o32 = torch.empty(B_, N_q, H_q, 128, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_prefill_window(s1.q, s1.k, s1.v_fp8, s1.delta, s1.stats, 0.5, window, sinks, w.softmax_scale, out, o32, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    rounded(out, o32)
    Q, K = plain.tile_rows(s1.q), plain.tile_rows(s1.k)
    V = plain.E4M3[s1.v_fp8.cpu().numpy().reshape(B_, H_kv, -1, 128)[:, :, :N_kv]]
    D = plain.bf16(s1.delta)[:, :, :N_kv]
    pos = np.arange(N_q) + N_kv - N_q
    for b in range(B_):
        check_rows(Q[b], K[b], V[b], D[b], o32[b].cpu().numpy(), pos, window, sinks, plain.lam_of(s1.stats, b, w.softmax_scale), 0.5,
                   (H_q, H_kv), b)
    if window >= N_kv:
        with arrangement(0):
            full, f32, _ = B.prefill(s1, True, w.softmax_scale, want_f32=True)
        assert torch.equal(full, out) and torch.equal(f32, o32)


def test_prefill_window_without_compensation_and_in_the_other_arrangement():
    """No Delta_S; and mpfa_set_prefill_arrangement does not concern the call."""
    B = binding()
    w = wl.prefill_workload("pw", 970, 1, 500, 4, 2, True)
    s1 = B.stage1(w.q.cuda(), w.k.cuda(), w.v.cuda(), smooth=False)
    outs = []
    for a in (0, 1):
        with arrangement(a):
            o32 = torch.empty(1, 500, 4, 128, device="cuda")
            out = torch.empty(1, 500, 4, 128, dtype=torch.bfloat16, device="cuda")
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            B.mpfa_prefill_window(s1.q, s1.k, s1.v_fp8, None, s1.stats, 1.0, 150, 2, w.softmax_scale, out, o32, status)
            torch.cuda.synchronize()
        assert int(status) == 0
        outs.append(o32)
    assert torch.equal(*outs)
    V = plain.E4M3[s1.v_fp8.cpu().numpy().reshape(1, 2, -1, 128)[:, :, :500]]
    check_rows(plain.tile_rows(s1.q)[0], plain.tile_rows(s1.k)[0], V[0], np.zeros((4, 500)), outs[0][0].cpu().numpy(), np.arange(500), 150, 2,
               plain.lam_of(s1.stats, 0, w.softmax_scale), 1.0, (4, 2), "direct")


@pytest.mark.parametrize("lens,q_lens,N_q,H_q,H_kv,window,sinks", [
    ([300, 129, 513], None, 129, 4, 2, 100, 4),
    ([64, 1, 200], [64, 1, 0], 70, 8, 2, 30, 0),           # chunks of several lengths, one of them empty
    ([2000, 900], [150, 128], 150, 8, 1, 333, 70),
    ([4700], None, 130, 2, 2, 4200, 90),                   # 34 blocks and more: accumulated in runs
    ([700, 650], [1, 200], 200, 10, 2, 1, 1),
    ([1500, 1500], None, 300, 4, 1, (1 << 31) - 1, 0),
])
def test_prefill_paged_window(lens, q_lens, N_q, H_q, H_kv, window, sinks):
    """Pages that no query of the request sees are given away first."""
    B = binding()
    st = state(980 + N_q, lens, H_q, H_kv, v_scale=0.5)
    nb = len(lens)
    w = wl.decode_workload("bounded", 980 + N_q, nb, H_q, H_kv, 1, max(lens), seq_lens=lens)
    q4 = B.Fp4Tensor.empty(nb, H_q, N_q)
    B.mpfa_quantize_qk(w.q_sample[:, :N_q].contiguous().cuda(), None, B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    ql = [N_q] * nb if q_lens is None else q_lens
    table = st.page_table.clone()
    there = []
    for b, L in enumerate(lens):
        # without queries a request needs no page at all
        there.append([i for i in range(-(-L // 64)) if ql[b] and (i * 64 < sinks or i * 64 + 63 > L - ql[b] - window)])
        for i in set(range(table.shape[1])) - set(there[b]):
            table[b, i] = (-5, 10 ** 9)[i % 2]
    out = torch.empty(nb, N_q, H_q, 128, dtype=torch.bfloat16, device="cuda")
    o32 = torch.empty(nb, N_q, H_q, 128, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ql_t = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    B.mpfa_prefill_paged_window(q4, st.kv, table, st.seq_lens, st.stats, 0.5, window, sinks, st.softmax_scale, out, o32, status, ql_t)
    torch.cuda.synchronize()
    assert int(status) == 0
    rounded(out, o32)
    Q = plain.tile_rows(q4)
    for b, L in enumerate(lens):
        got = o32[b].cpu().numpy()
        assert not got[ql[b]:].any()
        if ql[b]:
            K, V, D = plain.cached(st.kv, table[b].cpu().numpy(), L, there[b])
            check_rows(Q[b, :, :ql[b]], K, V, D, got[:ql[b]], np.arange(ql[b]) + L - ql[b], window, sinks,
                       plain.lam_of(st.stats, b, st.softmax_scale), 0.5, (H_q, H_kv), b)


# ------------------------------------------------------------------------------------------------------------------ weights
def weights_decode(st, weights, out=None, o32=None):
    B = binding()
    out = torch.empty_like(st.out) if out is None else out
    o32 = torch.empty_like(st.out_f32) if o32 is None else o32
    ws = B.decode_weights_workspace(st.q4.B, st.kv.H_q, st.kv.H_kv, st.page_table.shape[1])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_decode_weights(st.q4, st.kv, st.page_table, st.seq_lens, st.stats, st.v_scale, st.softmax_scale, weights, out, o32, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    return out, o32


def plain_weights(st, b):
    """[H_kv, L]"""
    L, G = int(st.seq_lens[b]), st.kv.H_q // st.kv.H_kv
    K, V, D = plain.cached(st.kv, st.page_table[b].cpu().numpy(), L)
    lam, q = plain.lam_of(st.stats, b, st.softmax_scale), plain.tile_rows(st.q4)
    S = np.stack([q[b, h, 0] @ K[h // G].T + D[h] for h in range(st.kv.H_q)])
    P = np.exp2(lam * (S - S.max(1, keepdims=True)))
    return (P / P.sum(1, keepdims=True)).reshape(st.kv.H_kv, G, L).sum(1)


@pytest.mark.parametrize("H_q,H_kv", [(4, 4), (4, 2), (6, 2), (8, 2), (10, 2), (12, 2), (14, 2), (16, 2)])
@pytest.mark.parametrize("lens", [[1, 0, 64, 129, 1025, 2600], [700, 5], [5000, 4097]])
def test_weights_of_every_group(H_q, H_kv, lens):
    """Outputs are decode's; each key's sum grows by its weights: each off by NEAR twice (exponent, l), and one rounding of the sum."""
    from paper_2609_33135_b200 import decode_cache
    st = state(1000 + H_q, lens, H_q, H_kv)
    slots = st.page_table.shape[1] * 64
    old = torch.rand(len(lens), H_kv, slots, generator=torch.Generator().manual_seed(5)).cuda()
    weights = old.clone()
    decode_cache.decode_step(st)
    out, o32 = weights_decode(st, weights)
    assert torch.equal(out, st.out) and torch.equal(o32, st.out_f32)
    for b, L in enumerate(lens):
        assert torch.equal(weights[b, :, L:], old[b, :, L:])
        if L:
            want = plain_weights(st, b)
            first, got = old[b, :, :L].cpu().numpy().astype(np.float64), weights[b, :, :L].cpu().numpy()
            close(got, first + want, 2 * plain.NEAR * want + 2.0 ** -24 * (first + want) * (1 + 2.0 ** -20), (b, L))


@pytest.mark.parametrize("offset,stride", [(0, 704), (1, 704), (0, 705), (3, 707)])
def test_weights_need_no_alignment(offset, stride):
    st = state(1020, [700, 333], 8, 2)
    flat = torch.zeros(2 * 2 * stride + 8, device="cuda")
    weights = flat[offset:offset + 4 * stride].view(2, 2, stride)
    weights_decode(st, weights)
    for b, L in enumerate((700, 333)):
        want = plain_weights(st, b)
        close(weights[b, :, :L].cpu().numpy(), want, (2 * plain.NEAR + 2.0 ** -24) * want, b)
        assert not weights[b, :, L:].any()
    assert not flat[:offset].any() and not flat[offset + 4 * stride:].any()


def test_weights_of_wide_tables_and_past_the_table():
    """A table far wider than the requests are long (few blocks for many chunks), and a length that the table cannot hold."""
    B = binding()
    st = state(1021, [900, 40, 2000], 4, 2)
    wide = torch.full((3, 4096), -1, dtype=torch.int32, device="cuda")
    wide[:, :st.page_table.shape[1]] = st.page_table
    narrow = torch.zeros(3, 2, st.page_table.shape[1] * 64, device="cuda")
    out, _ = weights_decode(st, narrow)
    st.page_table = wide
    weights = torch.zeros(3, 2, 4096 * 64, device="cuda")
    again, _ = weights_decode(st, weights)
    # many partitions are merged in another order of sums than few
    assert torch.allclose(out.float(), again.float(), rtol=2.0 ** -7, atol=0)
    n = narrow.shape[2]
    assert torch.allclose(weights[:, :, :n], narrow, rtol=2.0 ** -20, atol=0) and not weights[:, :, n:].any()
    full = state(1022, [640, 640], 4, 2)
    a, b = torch.zeros(2, 2, 640, device="cuda"), torch.zeros(2, 2, 640, device="cuda")
    weights_decode(full, a)
    full.seq_lens[0] = 2 ** 31 - 1
    weights_decode(full, b)
    assert torch.equal(a, b)
    assert B is not None


# ------------------------------------------------------------------------------------------------------------------ eviction
def pool(seed, lens, H_q, H_kv, spare, delta=True):
    """A cache of random bytes (the call moves them and computes nothing), a shuffled table and pages for the result."""
    B = binding()
    g = torch.Generator().manual_seed(seed)
    per = [-(-max(L, 1) // 64) for L in lens]
    n = sum(per) + spare + 3
    order = torch.randperm(n, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(per)), -7, dtype=torch.int32)
    at = 0
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        at += k
    def raw(*s):
        return torch.randint(0, 256, s, generator=g, dtype=torch.uint8).cuda()
    kv = B.PagedKV(raw(n, H_kv, 4096), raw(n, H_kv, 512), raw(n, H_kv, 8192),
                   torch.randn(n, H_q, 64, generator=g).bfloat16().cuda() if delta else None, n, H_q, H_kv)
    return kv, table.cuda(), order[at:at + spare].cuda()


def logical(kv, page):
    from layouts import paged_delta_to_logical, paged_k_to_logical, paged_v_to_logical
    k, v = paged_k_to_logical(kv.k_codes[page].cpu().numpy()), paged_v_to_logical(kv.v_fp8[page].cpu().numpy())
    d = None if kv.delta is None else paged_delta_to_logical(kv.delta[page].view(torch.int16).cpu().numpy(), kv.H_q // kv.H_kv)
    return k, kv.k_sf[page].cpu().numpy().reshape(kv.H_kv, 64, 8), v, d


def evict(kv, table, lens, weights, keep, sinks, recent, new_table, stride=None):
    B = binding()
    nb = table.shape[0]
    kept = torch.full((nb, kv.H_kv, keep), 77, dtype=torch.int32, device="cuda")
    new_lens = torch.full((nb,), 77, dtype=torch.int32, device="cuda")
    new_weights = torch.full((nb, kv.H_kv, stride or keep), 77.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_evict_paged(kv, table, lens, weights, keep, sinks, recent, new_table, kept, new_lens, new_weights, status)
    torch.cuda.synchronize()
    return kept, new_lens, new_weights, int(status)


def check_evicted(kv, before, table, lens, weights, keep, sinks, recent, new_table, kept, new_lens, new_weights, moved=True):
    G = kv.H_q // kv.H_kv
    written = set()
    for b, L in enumerate(lens):
        n = min(L, keep)
        assert int(new_lens[b]) == n
        for hk in range(kv.H_kv):
            want = plain.evicted(weights[b, hk].cpu().numpy(), L, keep, sinks, recent)
            assert np.array_equal(kept[b, hk, :n].cpu().numpy(), want), (b, hk)
            assert (kept[b, hk, n:] == -1).all() and not new_weights[b, hk, n:].any()
            assert np.array_equal(new_weights[b, hk, :n].cpu().numpy(), weights[b, hk].cpu().numpy()[want], equal_nan=True)
        written |= {int(p) for p in new_table[b, :-(-n // 64)]}
        if not moved:
            continue
        old = [logical(before, int(p)) for p in table[b, :max(1, -(-L // 64))]]
        for i in range(-(-n // 64)):
            k, s, v, d = logical(kv, int(new_table[b, i]))
            for hk in range(kv.H_kv):
                at = kept[b, hk, i * 64:min(i * 64 + 64, n)].cpu().numpy()
                c = len(at)
                assert np.array_equal(k[hk, :c], np.stack([old[a // 64][0][hk, a % 64] for a in at]))
                assert np.array_equal(s[hk, :c], np.stack([old[a // 64][1][hk, a % 64] for a in at]))
                assert np.array_equal(v[hk, :c], np.stack([old[a // 64][2][hk, a % 64] for a in at]))
                assert not k[hk, c:].any() and not s[hk, c:].any() and not v[hk, c:].any()
                for h in range(hk * G, hk * G + G) if d is not None else ():
                    assert np.array_equal(d[h, :c], [old[a // 64][3][h, a % 64] for a in at]) and not d[h, c:].any()
    rest = [p for p in range(kv.num_pages) if p not in written]
    for x, y in ((kv.k_codes, before.k_codes), (kv.k_sf, before.k_sf), (kv.v_fp8, before.v_fp8), (kv.delta, before.delta)):
        assert x is None or torch.equal(x[rest].view(torch.uint8 if x.dtype == torch.uint8 else torch.int16),
                                        y[rest].view(torch.uint8 if x.dtype == torch.uint8 else torch.int16))


def copy_of(kv):
    B = binding()
    return B.PagedKV(kv.k_codes.clone(), kv.k_sf.clone(), kv.v_fp8.clone(), None if kv.delta is None else kv.delta.clone(), kv.num_pages,
                     kv.H_q, kv.H_kv)


@pytest.mark.parametrize("lens,H_q,H_kv,keep,sinks,recent", [
    ([700, 100, 0, 333], 8, 2, 100, 4, 20),
    ([65, 64, 63, 1], 4, 4, 64, 0, 0),
    ([300, 2], 16, 2, 1, 0, 0),                # one token
    ([300, 301], 10, 2, 1, 1, 0),              # a sink and nothing else
    ([300, 301], 6, 2, 130, 100, 30),          # protected tokens only
    ([1500, 90], 8, 1, 129, 0, 129),           # the newest only
    ([2000], 14, 2, 1999, 4, 64),              # all but one
    ([900, 901], 4, 2, 700, 4, 0),
])
def test_eviction(lens, H_q, H_kv, keep, sinks, recent):
    per = -(-keep // 64)
    kv, table, spare = pool(1100 + keep, lens, H_q, H_kv, len(lens) * per)
    weights = torch.rand(len(lens), H_kv, table.shape[1] * 64 + 3, generator=torch.Generator().manual_seed(keep)).cuda()
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    before, new_table = copy_of(kv), spare.view(len(lens), per)
    kept, new_lens, new_weights, status = evict(kv, table, lens_t, weights, keep, sinks, recent, new_table, keep + 70)
    assert status == 0
    check_evicted(kv, before, table, lens, weights, keep, sinks, recent, new_table, kept, new_lens, new_weights)


def test_eviction_without_delta_and_with_spare_columns():
    kv, table, spare = pool(1150, [500, 400], 4, 2, 2 * 5, delta=False)
    weights = torch.rand(2, 2, table.shape[1] * 64).cuda()
    before = copy_of(kv)
    new_table = spare.view(2, 5)
    got = evict(kv, table, torch.tensor([500, 400], dtype=torch.int32, device="cuda"), weights, 190, 1, 1, new_table)
    assert got[3] == 0
    check_evicted(kv, before, table, [500, 400], weights, 190, 1, 1, new_table, *got[:3])


@pytest.mark.parametrize("kind", ["equal", "two", "zeros", "special", "dense", "negative"])
@pytest.mark.parametrize("L", [200, 5000, 20000, 60000])   # rows of one CTA, and of clusters of four and eight
def test_eviction_by_weights_that_are_alike(kind, L):
    """Ties, the lowest slot first; infinities and NaN; many weights that differ in their last bits only; more than fit shared memory."""
    keep, sinks, recent = L // 2 + 1, 3, 10
    g = torch.Generator().manual_seed(L)
    B = binding()
    per, pages = -(-keep // 64), -(-L // 64)
    kv = B.PagedKV.empty(pages + per, 2, 2)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    w = torch.rand(1, 2, pages * 64, generator=g)
    if kind == "equal":
        w.fill_(0.25)
    elif kind == "two":
        w = (w > 0.3).float()
    elif kind == "zeros":
        w = torch.where(w > 0.5, 0.0, -0.0)
    elif kind == "special":
        pick = torch.randint(0, 6, w.shape, generator=g)
        for i, x in enumerate((float("nan"), float("inf"), -float("inf"), 1e-42, -1e-42)):
            w[pick == i] = x
        w[:, 1] = float("nan")
    elif kind == "dense":
        w = 1.0 + torch.randint(0, 40, w.shape, generator=g) * 2.0 ** -23
    else:
        w = w - 0.5
    w = w.cuda()
    new_table = torch.arange(pages, pages + per, dtype=torch.int32, device="cuda").view(1, -1)
    got = evict(kv, table, torch.tensor([L], dtype=torch.int32, device="cuda"), w, keep, sinks, recent, new_table)
    assert got[3] == 0
    check_evicted(kv, copy_of(kv), table, [L], w, keep, sinks, recent, new_table, *got[:3], moved=False)


def test_eviction_reports_bad_pages():
    B = binding()
    kv, table, spare = pool(1160, [300, 300], 4, 2, 2 * 4)
    weights = torch.rand(2, 2, table.shape[1] * 64).cuda()
    lens = torch.tensor([300, 300], dtype=torch.int32, device="cuda")
    new_table = spare.view(2, 4).clone()
    before = copy_of(kv)
    table[0, 0] = kv.num_pages            # a source page: its tokens become zeros
    new_table[1, 1] = -1                  # a page to write: left out
    kept, new_lens, new_weights, status = evict(kv, table, lens, weights, 250, 70, 70, new_table)
    assert status == B.MPFA_DEV_BAD_PAGE
    assert new_lens.tolist() == [250, 250]
    k, s, v, d = logical(kv, int(new_table[0, 0]))
    assert not k.any() and not v.any() and not s.any() and not d.any()
    k, _, _, _ = logical(kv, int(new_table[1, 0]))
    assert np.array_equal(k, logical(before, int(table[1, 0]))[0])   # 64 sinks
    for b in range(2):
        for hk in range(2):
            assert np.array_equal(kept[b, hk].cpu().numpy(), plain.evicted(weights[b, hk].cpu().numpy(), 300, 250, 70, 70))


# ------------------------------------------------------------------------------------------------------------------ together
def test_a_bounded_request_from_prompt_to_eviction():
    """What a serving program does: the prompt in pages, tokens appended and decoded with their weights summed, the cache cut back to its
    budget, and on; the whole of it captured and replayed, on another stream than the current one."""
    B = binding()
    H_q, H_kv, L0, steps, keep = 8, 2, 500, 6, 400
    w = wl.decode_workload("together", 1200, 2, H_q, H_kv, 1, L0 + steps, seq_lens=[L0, L0 - 133])
    from paper_2609_33135_b200 import decode_cache

    def fresh():
        st = decode_cache.build_cache(w)
        pages = -(-(L0 + 2 * steps) // 64)
        # room for the appended tokens and for the pages after eviction
        n = st.kv.num_pages
        big = B.PagedKV.empty(n + 40, H_q, H_kv)
        for a, b in ((big.k_codes, st.kv.k_codes), (big.k_sf, st.kv.k_sf), (big.v_fp8, st.kv.v_fp8), (big.delta, st.kv.delta)):
            a[:n] = b
        table = torch.full((2, pages), -1, dtype=torch.int32, device="cuda")
        table[:, :st.page_table.shape[1]] = st.page_table
        free = iter(range(n, n + 40))
        for b in range(2):
            for i in range(-(-int(st.seq_lens[b]) // 64), pages):
                table[b, i] = next(free)
        new_table = torch.tensor([[next(free) for _ in range(-(-(keep + steps) // 64))] for _ in range(2)], dtype=torch.int32, device="cuda")
        st.kv, st.page_table = big, table
        return st, new_table

    k, v, q = (torch.randn(2 * steps, 2, 1, h, 128, generator=torch.Generator().manual_seed(s)).bfloat16().cuda()
               for s, h in ((1, H_kv), (2, H_kv), (3, H_q)))

    def serve(st, new_table):
        flags = B.MPFA_SMOOTH
        lens, slots = st.seq_lens.clone(), st.page_table.shape[1] * 64
        weights = torch.zeros(2, H_kv, slots, device="cuda")
        kept = torch.empty(2, H_kv, keep, dtype=torch.int32, device="cuda")
        new_lens, new_weights = torch.empty_like(lens), torch.empty(2, H_kv, slots, device="cuda")
        ws = B.decode_weights_workspace(2, H_q, H_kv, st.page_table.shape[1])
        wws = B.decode_window_workspace(2, H_q, H_kv, st.page_table.shape[1], 100, 4)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        outs = [torch.empty(2, H_q, 128, dtype=torch.bfloat16, device="cuda") for _ in range(3 * steps)]

        def step(i, table, lens, weights, out):
            B.mpfa_append_kv_paged(k[i], v[i], H_q, flags, st.stats, 1.0, st.kv, table, lens)
            lens += 1
            B.mpfa_quantize_qk(q[i], None, flags | B.MPFA_STATS_FROZEN, st.stats, st.q4, None, None, None)
            B.mpfa_decode_weights(st.q4, st.kv, table, lens, st.stats, 1.0, st.softmax_scale, weights, out, None, ws, status)

        for i in range(steps):
            step(i, st.page_table, lens, weights, outs[i])
            B.mpfa_decode_window(st.q4, st.kv, st.page_table, lens, st.stats, 1.0, 100, 4, st.softmax_scale, outs[2 * steps + i], None, wws, status)
        B.mpfa_evict_paged(st.kv, st.page_table, lens, weights, keep, 4, 50, new_table, kept, new_lens, new_weights, status)
        wide = torch.full_like(st.page_table, -1)
        wide[:, :new_table.shape[1]] = new_table
        for i in range(steps):
            step(steps + i, wide, new_lens, new_weights, outs[steps + i])
        return outs, weights, kept, new_lens, new_weights, status, wide, lens

    st, new_table = fresh()
    eager = serve(st, new_table)
    torch.cuda.synchronize()
    assert int(eager[5]) == 0 and eager[3].tolist() == [keep + steps, L0 - 133 + 2 * steps]
    # the last step of the evicted cache against the plain statement, over the tokens that each head kept
    kv, lens = st.kv, eager[3]
    qn = plain.tile_rows(st.q4)
    for b in range(2):
        L = int(lens[b])
        K, V, D = plain.cached(kv, eager[6][b].cpu().numpy(), L)
        lam = plain.lam_of(st.stats, b, st.softmax_scale)
        for h in range(H_q):
            want, room, _, _ = plain.attend(qn[b, h], K[h // 4], V[h // 4], D[h], np.ones((1, L), bool), lam, 1.0, 8)
            close(eager[0][2 * steps - 1][b, h].float().cpu().numpy(), want[0], room[0] + 2.0 ** -8 * np.abs(want[0]), (b, h))
    # each step gives every kv head of a request as much as it has q heads
    total = eager[1].sum(2).cpu().numpy()
    assert np.allclose(total, steps * 4, rtol=2.0 ** -13)

    again, table2 = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(again, table2)   # first calls, outside a capture
    torch.cuda.synchronize()
    third, table3 = fresh()
    kept_lens = third.seq_lens.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        replayed = serve(third, table3)
    for _ in range(2):
        third.seq_lens.copy_(kept_lens)
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager[0], replayed[0]):
        assert torch.equal(a, b)
    for i in (1, 2, 3, 4):
        assert torch.equal(eager[i], replayed[i])


def test_two_streams_with_workspaces_of_their_own():
    sts = [state(1210 + i, [3000, 200, 1100], 8, 2) for i in range(2)]
    alone = [window_decode(st, 900, 4)[0] for st in sts]
    B = binding()
    streams = [torch.cuda.Stream() for _ in sts]
    bufs = [(B.decode_window_workspace(3, 8, 2, st.page_table.shape[1], 900, 4), torch.empty_like(st.out),
             torch.zeros(1, dtype=torch.int32, device="cuda")) for st in sts]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, s, (ws, out, status) in zip(sts, streams, bufs):
            with torch.cuda.stream(s):
                B.mpfa_decode_window(st.q4, st.kv, st.page_table, st.seq_lens, st.stats, 1.0, 900, 4, st.softmax_scale, out, None, ws, status)
    torch.cuda.synchronize()
    for want, (_, out, status) in zip(alone, bufs):
        assert int(status) == 0 and torch.equal(out, want)


def test_the_cache_module_serves_bounded_requests():
    """decode_cache's own calls: a window, sums of the weights, and eviction after which the request goes on with its new pages."""
    from paper_2609_33135_b200 import decode_cache
    B = binding()
    st = state(1220, [900, 300], 8, 2)
    want, _ = window_decode(st, 200, 5)
    assert torch.equal(decode_cache.decode_step(st, window=200, sinks=5), want)
    sums = decode_cache.attention_sums(st)
    decode_cache.decode_step(st, weights=sums)
    pages, n, big = 5, st.kv.num_pages, B.PagedKV.empty(st.kv.num_pages + 10, 8, 2)
    for new, old in ((big.k_codes, st.kv.k_codes), (big.k_sf, st.kv.k_sf), (big.v_fp8, st.kv.v_fp8), (big.delta, st.kv.delta)):
        new[:n] = old
    st.kv = big
    new_pages = torch.arange(n, n + 10, dtype=torch.int32, device="cuda").view(2, pages)
    kept, new_sums = decode_cache.evict(st, sums, 300, 4, 100, new_pages)
    assert st.seq_lens.tolist() == [300, 300] and new_sums.shape == (2, 2, 320)
    for hk in range(2):
        assert kept[0, hk].tolist() == plain.evicted(sums[0, hk].cpu().numpy(), 900, 300, 4, 100).tolist()
        assert kept[1, hk].tolist() == list(range(300))
    before = new_sums.clone()
    decode_cache.decode_step(st, weights=new_sums)
    torch.cuda.synchronize()
    assert int(st.status) == 0
    assert torch.allclose((new_sums - before).sum(2), torch.full((2, 2), 4.0, device="cuda"), rtol=2.0 ** -12)


def test_lengths_below_zero_count_as_none():
    B = binding()
    st = state(1230, [300, 200, 100], 4, 2)
    want, _ = window_decode(st, 50, 2)
    st.seq_lens[1] = -(2 ** 31)
    out, o32 = window_decode(st, 50, 2)
    assert torch.equal(out[0::2], want[0::2]) and not o32[1].any()
    weights = torch.zeros(3, 2, st.page_table.shape[1] * 64, device="cuda")
    out, o32 = weights_decode(st, weights)
    assert not o32[1].any() and not weights[1].any() and bool(weights[0, :, :300].all())
    q4 = B.Fp4Tensor.empty(3, 4, 9)
    B.mpfa_quantize_qk(torch.randn(3, 9, 4, 128, device="cuda").bfloat16(), None, B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    o = torch.full((3, 9, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_prefill_paged_window(q4, st.kv, st.page_table, st.seq_lens, st.stats, 1.0, 50, 2, st.softmax_scale, o, None, status)
    assert int(status) == 0 and not o[1].any() and bool(o[0].any())
    kv, table, spare = pool(1231, [300, 200], 4, 2, 4)
    lens = torch.tensor([-5, 200], dtype=torch.int32, device="cuda")
    w = torch.rand(2, 2, table.shape[1] * 64).cuda()
    kept, new_lens, new_weights, status = evict(kv, table, lens, w, 100, 4, 4, spare.view(2, 2))
    assert status == 0 and new_lens.tolist() == [0, 100] and (kept[0] == -1).all() and not new_weights[0].any()


def test_nothing_is_written_outside_the_buffers():
    """Every buffer that these calls write, workspaces of exactly the size that is asked for among them, cut out of one arena with guard bands
    whose bytes have to stay."""
    B = binding()
    arena, cuts, at = torch.full((64 << 20,), 0xA5, dtype=torch.uint8, device="cuda"), [], [0]

    def cut(n, dtype=torch.uint8, shape=None):
        begin = (at[0] + 4096 + 1023) // 1024 * 1024
        at[0] = begin + n
        cuts.append((begin, begin + n))
        t = arena[begin:begin + n].view(dtype)
        return t if shape is None else t.view(shape)

    def intact():
        torch.cuda.synchronize()
        last = 0
        for a, b in cuts + [(arena.numel(), arena.numel())]:
            assert bool((arena[last:a] == 0xA5).all()), (last, a)
            last = b

    st = state(1240, [2500, 1, 130], 10, 2)
    P, n = st.page_table.shape[1], st.kv.num_pages
    status = cut(4, torch.int32)
    status.zero_()
    out, o32 = cut(3 * 10 * 256, torch.bfloat16, (3, 10, 128)), cut(3 * 10 * 512, torch.float32, (3, 10, 128))
    L = B.lib()
    ws = cut(L.mpfa_decode_window_workspace_bytes(3, 10, 2, P, 1100, 200))
    B.mpfa_decode_window(st.q4, st.kv, st.page_table, st.seq_lens, st.stats, 1.0, 1100, 200, st.softmax_scale, out, o32, ws, status)
    intact()
    ws = cut(L.mpfa_decode_weights_workspace_bytes(3, 10, 2, P))
    weights = cut(3 * 2 * P * 64 * 4, torch.float32, (3, 2, P * 64))
    weights.zero_()
    B.mpfa_decode_weights(st.q4, st.kv, st.page_table, st.seq_lens, st.stats, 1.0, st.softmax_scale, weights, out, o32, ws, status)
    intact()
    keep, per = 333, 6
    kv = B.PagedKV(cut((n + 3 * per) * 2 * 4096, shape=(-1, 2, 4096)), cut((n + 3 * per) * 2 * 512, shape=(-1, 2, 512)),
                   cut((n + 3 * per) * 2 * 8192, shape=(-1, 2, 8192)), cut((n + 3 * per) * 10 * 128, torch.bfloat16, (-1, 10, 64)), n + 3 * per, 10, 2)
    for new, old in ((kv.k_codes, st.kv.k_codes), (kv.k_sf, st.kv.k_sf), (kv.v_fp8, st.kv.v_fp8), (kv.delta, st.kv.delta)):
        new[:n] = old
    new_table = torch.arange(n, n + 3 * per, dtype=torch.int32, device="cuda").view(3, per)
    kept, new_lens = cut(3 * 2 * keep * 4, torch.int32, (3, 2, keep)), cut(12, torch.int32)
    new_weights = cut(3 * 2 * 335 * 4, torch.float32, (3, 2, 335))
    B.mpfa_evict_paged(kv, st.page_table, st.seq_lens, weights, keep, 4, 50, new_table, kept, new_lens, new_weights, status)
    intact()
    q4 = B.Fp4Tensor.empty(3, 10, 131)
    B.mpfa_quantize_qk(torch.randn(3, 131, 10, 128, device="cuda").bfloat16(), None, B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    rows, r32 = cut(3 * 131 * 10 * 256, torch.bfloat16, (3, 131, 10, 128)), cut(3 * 131 * 10 * 512, torch.float32, (3, 131, 10, 128))
    B.mpfa_prefill_paged_window(q4, kv, new_table, new_lens, st.stats, 1.0, 70, 9, st.softmax_scale, rows, r32, status)
    intact()
    w = wl.prefill_workload("guards", 1241, 1, 300, 10, 2, True)
    s1 = B.stage1(w.q.cuda(), w.k.cuda(), w.v.cuda())
    B.mpfa_prefill_window(s1.q, s1.k, s1.v_fp8, s1.delta, s1.stats, 1.0, 70, 9, w.softmax_scale, cut(300 * 2560, torch.bfloat16),
                          cut(300 * 5120, torch.float32), status)
    intact()
    assert int(status) == 0 and new_lens.tolist() == [333, 1, 130] and at[0] < arena.numel()


def test_without_compensation_on_pages():
    """A cache without a Delta_S pool: decode with a window, decode with weights, a chunk under a window."""
    B = binding()
    st = state(1250, [1300, 77], 10, 2, v_scale=2.0, smooth=False)
    assert st.kv.delta is None
    out, o32 = window_decode(st, 333, 40)
    rounded(out, o32)
    check_window_decode(st, 333, 40, o32)
    weights = torch.zeros(2, 2, st.page_table.shape[1] * 64, device="cuda")
    weights_decode(st, weights)
    for b, L in enumerate((1300, 77)):
        want = plain_weights(st, b)
        close(weights[b, :, :L].cpu().numpy(), want, (2 * plain.NEAR + 2.0 ** -24) * want, b)
    q4 = B.Fp4Tensor.empty(2, 10, 60)
    B.mpfa_quantize_qk(torch.randn(2, 60, 10, 128, generator=torch.Generator().manual_seed(3)).bfloat16().cuda(), None, B.MPFA_STATS_FROZEN,
                       st.stats, q4, None, None, None)
    o32, status = torch.empty(2, 60, 10, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_prefill_paged_window(q4, st.kv, st.page_table, st.seq_lens, st.stats, 2.0, 200, 3, st.softmax_scale,
                                torch.empty(2, 60, 10, 128, dtype=torch.bfloat16, device="cuda"), o32, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    Q = plain.tile_rows(q4)
    for b, L in enumerate((1300, 77)):
        K, V, D = plain.cached(st.kv, st.page_table[b].cpu().numpy(), L)
        check_rows(Q[b], K, V, D, o32[b].cpu().numpy(), np.arange(60) + L - 60, 200, 3, plain.lam_of(st.stats, b, st.softmax_scale), 2.0, (10, 2), b)


@pytest.mark.parametrize("seed", range(12))
def test_windows_drawn(seed):
    """Drawn lengths, windows, sinks and groups, decode and a chunk of the same requests."""
    B, r = binding(), np.random.RandomState(seed)
    H_q, H_kv = [(4, 2), (8, 1), (6, 2), (5, 1)][seed % 4]
    lens = [int(x) for x in np.exp(r.uniform(0, np.log(2400), 3))]
    window, sinks, N_q = int(np.exp(r.uniform(0, np.log(2500)))), int(r.choice([0, 1, 5, 64, 100, 129, 400])), int(r.randint(1, 300))
    st = state(1300 + seed, lens, H_q, H_kv, v_scale=0.5)
    out, o32 = window_decode(st, window, sinks)
    rounded(out, o32)
    check_window_decode(st, window, sinks, o32)
    q_lens = [min(N_q, L) for L in lens]
    q4 = B.Fp4Tensor.empty(3, H_q, N_q)
    B.mpfa_quantize_qk(torch.randn(3, N_q, H_q, 128, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda(), None,
                       B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    o32, status = torch.empty(3, N_q, H_q, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_prefill_paged_window(q4, st.kv, st.page_table, st.seq_lens, st.stats, 0.5, window, sinks, st.softmax_scale,
                                torch.empty(3, N_q, H_q, 128, dtype=torch.bfloat16, device="cuda"), o32, status,
                                torch.tensor(q_lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(status) == 0
    Q = plain.tile_rows(q4)
    for b, L in enumerate(lens):
        K, V, D = plain.cached(st.kv, st.page_table[b].cpu().numpy(), L)
        n = q_lens[b]
        check_rows(Q[b, :, :n], K, V, D, o32[b, :n].cpu().numpy(), np.arange(n) + L - n, window, sinks, plain.lam_of(st.stats, b, st.softmax_scale),
                   0.5, (H_q, H_kv), b)
        assert not o32[b, n:].any()


def test_pools_of_more_than_four_gigabytes():
    """Slabs whose byte offsets do not fit 32 bits: the pages of a small cache moved to the end of a large pool."""
    B = binding()
    st = state(1400, [500, 333], 32, 8)
    window, wo32 = window_decode(st, 200, 70)
    sums = torch.zeros(2, 8, st.page_table.shape[1] * 64, device="cuda")
    full, _ = weights_decode(st, sums)
    small, n = st.kv, 66000                                      # 66000 x 8 x 8192 bytes of V
    used = small.num_pages
    big = B.PagedKV(*(torch.empty(n, *t.shape[1:], dtype=t.dtype, device="cuda") for t in (small.k_codes, small.k_sf, small.v_fp8, small.delta)),
                    n, 32, 8)
    for new, old in ((big.k_codes, small.k_codes), (big.k_sf, small.k_sf), (big.v_fp8, small.v_fp8), (big.delta, small.delta)):
        new[n - used:] = old
    st.kv, st.page_table = big, torch.where(st.page_table >= 0, st.page_table + (n - used), st.page_table)
    assert torch.equal(window_decode(st, 200, 70)[0], window)
    again = torch.zeros_like(sums)
    assert torch.equal(weights_decode(st, again)[0], full) and torch.equal(again, sums)
    new_table = torch.arange(n - used - 10, n - used, dtype=torch.int32, device="cuda").view(2, 5)
    kept, new_lens, _, status = evict(big, st.page_table, st.seq_lens, sums, 300, 4, 32, new_table)
    assert status == 0 and new_lens.tolist() == [300, 300]
    for b in range(2):
        old = [logical(big, int(p)) for p in st.page_table[b, :-(-int(st.seq_lens[b]) // 64)]]
        k, s, v, d = logical(big, int(new_table[b, 4]))
        for hk in range(8):
            for i, a in enumerate(kept[b, hk, 256:].tolist()):
                assert np.array_equal(v[hk, i], old[a // 64][2][hk, a % 64]) and np.array_equal(k[hk, i], old[a // 64][0][hk, a % 64])
                assert np.array_equal(s[hk, i], old[a // 64][1][hk, a % 64]) and d[hk * 4 + 3, i] == old[a // 64][3][hk * 4 + 3, a % 64]
    q4 = B.Fp4Tensor.empty(2, 32, 40)
    B.mpfa_quantize_qk(torch.randn(2, 40, 32, 128, generator=torch.Generator().manual_seed(4)).bfloat16().cuda(), None,
                       B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    outs = []
    for kv, table in ((small, torch.where(st.page_table >= 0, st.page_table - (n - used), st.page_table)), (big, st.page_table)):
        o = torch.empty(2, 40, 32, 128, dtype=torch.bfloat16, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.mpfa_prefill_paged_window(q4, kv, table, st.seq_lens, st.stats, 1.0, 100, 9, st.softmax_scale, o, None, status)
        assert int(status) == 0
        outs.append(o)
    assert torch.equal(*outs)


@pytest.mark.parametrize("nb,H_kv,L,keep,sinks,recent,kind", [
    (1, 2, 400000, 1000, 4, 100, "rand"),         # a cluster's parts do not fit shared memory
    (1, 1, 400000, 399000, 0, 0, "equal"),
    (75, 2, 49300, 600, 1, 64, "rand"),           # too many rows for clusters, too long for shared memory
    (80, 2, 20000, 8000, 10, 5, "two"),           # too many rows for clusters
    (30, 2, 20000, 8000, 10, 5, "rand"),          # clusters of two
    (1, 1, 20000, 5000, 2000, 3000, "rand"),      # clusters, protected tokens only
    (1, 3, 20000, 19999, 7, 7, "rand"),
    (2, 2, 33000, 1, 0, 0, "equal"),
])
def test_eviction_of_long_rows(nb, H_kv, L, keep, sinks, recent, kind):
    """Rows that several CTAs share, or that do not fit where they are held; lengths differ within a batch, short ones and none among them.
    Tables share the source pages (they are only read)."""
    B = binding()
    pages, per = -(-L // 64), -(-keep // 64)
    kv = B.PagedKV(*(torch.zeros(pages + nb * per, H_kv, n, dtype=torch.uint8, device="cuda") for n in (4096, 512, 8192)), None, pages + nb * per, H_kv,
                   H_kv)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(nb, 1)
    new_table = torch.arange(pages, pages + nb * per, dtype=torch.int32, device="cuda").view(nb, per)
    g = torch.Generator().manual_seed(L + keep)
    w = torch.rand(nb, H_kv, pages * 64, generator=g)
    if kind == "equal":
        w.fill_(1.0)
    elif kind == "two":
        w = (w > 0.5).float()
    w = w.cuda()
    lens = [L if b % 4 == 0 else (0, keep, min(L, keep + 700))[b % 3] for b in range(nb)]
    got = evict(kv, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), w, keep, sinks, recent, new_table)
    assert got[3] == 0 and got[1].tolist() == [min(n, keep) for n in lens]
    for b in sorted({0, 1 % nb, 2 % nb, 3 % nb, nb - 1}):
        for hk in range(H_kv):
            want = plain.evicted(w[b, hk].cpu().numpy(), lens[b], keep, sinks, recent)
            assert np.array_equal(got[0][b, hk, :len(want)].cpu().numpy(), want), (b, hk)
            assert (got[0][b, hk, len(want):] == -1).all() and not got[2][b, hk, len(want):].any()
            assert np.array_equal(got[2][b, hk, :len(want)].cpu().numpy(), w[b, hk].cpu().numpy()[want])
    # every row is as long as its count says, ascending
    rows, n = got[0], torch.tensor([min(x, keep) for x in lens], device="cuda").view(-1, 1, 1)
    live = torch.arange(keep, device="cuda") < n
    assert bool(((rows >= 0) == live).all()) and bool(((rows[..., 1:] > rows[..., :-1]) | ~live[..., 1:]).all())


def test_eviction_of_long_rows_from_a_graph():
    """The form with clusters captured and replayed on other weights and lengths than it was captured with."""
    B = binding()
    L, keep, H_kv = 33000, 5000, 2
    pages, per = -(-L // 64), -(-keep // 64)
    kv = B.PagedKV.empty(pages + per, H_kv, H_kv)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    new_table = torch.arange(pages, pages + per, dtype=torch.int32, device="cuda").view(1, -1)
    w, lens = torch.rand(1, H_kv, pages * 64, device="cuda"), torch.tensor([L], dtype=torch.int32, device="cuda")
    kept, new_lens = torch.empty(1, H_kv, keep, dtype=torch.int32, device="cuda"), torch.empty_like(lens)
    new_weights, status = torch.empty(1, H_kv, keep, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def go():
        B.mpfa_evict_paged(kv, table, lens, w, keep, 4, 100, new_table, kept, new_lens, new_weights, status)

    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for n in (L, 21000, 5000, 17):
        w.copy_(torch.rand(w.shape, generator=torch.Generator().manual_seed(n)))
        lens.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0 and new_lens.tolist() == [min(n, keep)]
        for hk in range(H_kv):
            want = plain.evicted(w[0, hk].cpu().numpy(), n, keep, 4, 100)
            assert np.array_equal(kept[0, hk, :len(want)].cpu().numpy(), want)
            assert np.array_equal(new_weights[0, hk, :len(want)].cpu().numpy(), w[0, hk].cpu().numpy()[want]) and not new_weights[0, hk, len(want):].any()
