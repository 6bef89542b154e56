"""GPU: the calls for bounded caches where callers, streams and caches are not the plain ones: host threads side by side, pages that are
missing, heads without a softmax, tables that grow, tensors of another stream, hidden values, more requests than the kernels hold lengths for."""
import threading

import numpy as np
import pytest
import torch

import bounded_plain as plain
import test_gpu_bounded as bounded
from paper_2609_33135_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def binding():
    from paper_2609_33135_b200 import binding as B
    return B


# ------------------------------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("pages", [(18, 256), (400, 4000)])   # one CTA to a row; clusters
def test_host_threads_evict_from_tables_of_different_widths(pages):
    """The interpreter's lock is released during a call, so the threads' launches mix.  The arguments are made once, which leaves the threads
    little else to do than to call."""
    B = binding()
    jobs = []
    for n in pages * 2:
        L, keep = n * 64, n * 32
        kv = B.PagedKV.empty(n + n // 2, 1, 1)
        table = torch.arange(n, dtype=torch.int32, device="cuda").view(1, -1)
        new_table = torch.arange(n, n + n // 2, dtype=torch.int32, device="cuda").view(1, -1)
        w = torch.rand(1, 1, L, generator=torch.Generator().manual_seed(n)).cuda()
        jobs.append((kv, table, torch.tensor([L], dtype=torch.int32, device="cuda"), w, keep, 4, 16, new_table,
                     torch.empty(1, 1, keep, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda"),
                     torch.empty(1, 1, keep, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    call, start, answers = B.lib().packed_mpfa_evict_paged, threading.Barrier(len(jobs)), []

    def serve(kv, table, lens, w, keep, sinks, recent, new_table, kept, new_lens, new_weights, status, stream):
        at = [t.data_ptr() for t in (table, lens, w, new_table, kept, new_lens, new_weights, status)]
        args = (kv.packed_paged(), at[0], 1, table.shape[1], at[1], at[2], w.shape[2], keep, sinks, recent, at[3], new_table.shape[1], at[4], at[5],
                at[6], keep, at[7], stream.cuda_stream)
        start.wait()
        for i in range(4000):
            rc = call(*args)
            if rc or i % 500 == 499:
                answers.append(rc)
                stream.synchronize()   # few enough on the way that a launch does not wait for room

    threads = [threading.Thread(target=serve, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not any(answers), sum(map(bool, answers))
    for kv, table, lens, w, keep, sinks, recent, _, kept, new_lens, _, status, _ in jobs:
        assert int(status) == 0 and new_lens.tolist() == [keep]
        assert np.array_equal(kept[0, 0].cpu().numpy(), plain.evicted(w[0, 0].cpu().numpy(), w.shape[2], keep, sinks, recent))


# ------------------------------------------------------------------------------------------------------------------ weights
def sums_of(st, table, old):
    """One step that adds to a copy of `old`: (sums, out, out_f32, status)."""
    B = binding()
    weights, out, o32 = old.clone(), torch.empty_like(st.out), torch.empty_like(st.out_f32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_decode_weights(st.q4, st.kv, table, st.seq_lens, st.stats, st.v_scale, st.softmax_scale, weights, out, o32,
                          B.decode_weights_workspace(st.q4.B, st.kv.H_q, st.kv.H_kv, table.shape[1]), status)
    torch.cuda.synchronize()
    return weights, out, o32, int(status)


def random_sums(st, seed):
    shape = st.q4.B, st.kv.H_kv, st.page_table.shape[1] * 64
    return torch.rand(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


def close_sums(got, old, want, what):
    """As for whole caches: each weight off by NEAR twice (exponent, l), and one rounding of the sum."""
    old, got = old.cpu().numpy().astype(np.float64), got.cpu().numpy()
    bounded.close(got, old + want, 2 * plain.NEAR * want + 2.0 ** -24 * (old + want) * (1 + 2.0 ** -20), what)


def set_delta(kv, page, h, t, value):
    kv.delta[page, h, ((t // 8) ^ (h % (kv.H_q // kv.H_kv))) * 8 + t % 8] = value


@pytest.mark.parametrize("H_q,H_kv", [(4, 4), (4, 2), (8, 1)])
@pytest.mark.parametrize("value", [-float("inf"), float("nan"), float("inf")])
@pytest.mark.parametrize("lens", [[300, 64], [2600, 1500], [5000, 4097]])   # one partition; a few; many
def test_heads_without_a_softmax_add_nothing(H_q, H_kv, value, lens):
    """All logits of a kv head's q heads -infinity, NaN or +infinity: no output, and no trace in the sums."""
    from paper_2609_33135_b200 import decode_cache
    st, G = bounded.state(1520 + H_q, lens, H_q, H_kv), H_q // H_kv
    bad = H_kv - 1
    for h in range(bad * G, bad * G + G):
        for i in range(-(-lens[0] // 64)):
            st.kv.delta[int(st.page_table[0, i]), h] = value
    old = random_sums(st, 2)
    weights, out, o32, status = sums_of(st, st.page_table, old)
    decode_cache.decode_step(st)
    torch.cuda.synchronize()
    assert status == 0 and torch.equal(out, st.out) and torch.equal(o32, st.out_f32)
    assert not o32[0, bad * G:].any() and torch.equal(weights[0, bad], old[0, bad])
    for b, L in enumerate(lens):
        want = bounded.plain_weights(st, b)
        heads = [hk for hk in range(H_kv) if b or hk != bad]
        if heads:
            close_sums(weights[b, heads, :L], old[b, heads, :L], want[heads], b)


def test_logits_that_are_no_numbers_leave_the_sums_numbers():
    """One NaN scale: the heads that see the key have no softmax.  A partition of nothing else is left out, and its keys receive nothing."""
    lens, H_q, H_kv = [300, 2600], 8, 4
    st = bounded.state(1530, lens, H_q, H_kv)
    st.kv.k_sf[int(st.page_table[0, 0]), 0, 5 * 8:5 * 8 + 8] = 0x7F
    for i in range(16, 32):
        st.kv.k_sf[int(st.page_table[1, i]), 2] = 0x7F
    old = random_sums(st, 3)
    weights, out, o32, status = sums_of(st, st.page_table, old)
    assert status == 0 and bool(torch.isfinite(weights).all())
    assert not o32[0, :2].any() and torch.equal(weights[0, 0], old[0, 0])
    assert torch.equal(weights[1, 2, 1024:2048], old[1, 2, 1024:2048])
    lam, q = plain.lam_of(st.stats, 1, st.softmax_scale), plain.tile_rows(st.q4)
    K, V, D = plain.cached(st.kv, st.page_table[1].cpu().numpy(), 2600)
    there = np.r_[0:1024, 2048:2600]
    want = np.zeros(len(there))
    for h in (4, 5):
        S = q[1, h, 0] @ K[2, there].T + D[h, there]
        P = np.exp2(lam * (S - S.max()))
        want += P / P.sum()
    close_sums(weights[1, 2, there], old[1, 2, there], want, "beside the partition")
    for b, heads in ((0, [1, 2, 3]), (1, [0, 1, 3])):
        close_sums(weights[b, heads, :lens[b]], old[b, heads, :lens[b]], bounded.plain_weights(st, b)[heads], b)


@pytest.mark.parametrize("H_q,H_kv", [(4, 4), (8, 2), (10, 2), (16, 2)])
def test_keys_on_missing_pages_receive_no_weight(H_q, H_kv):
    """They are in no softmax either: the others' weights, and the output, are those of the keys that are there."""
    B = binding()
    lens = [2600, 700, 64]
    st, G = bounded.state(1500 + H_q, lens, H_q, H_kv, v_scale=0.5), H_q // H_kv
    old = random_sums(st, 1)
    clean, clean_out, _, status = sums_of(st, st.page_table, old)
    assert status == 0
    table = st.page_table.clone()
    gone = {0: [3] + list(range(16, 32)) + [40], 1: [], 2: [0]}   # a page, a whole partition and the last page; none; all
    for b, pages in gone.items():
        for i in pages:
            table[b, i] = (-1, st.kv.num_pages, 2 ** 31 - 1)[i % 3]
    weights, out, o32, status = sums_of(st, table, old)
    assert status == B.MPFA_DEV_BAD_PAGE
    assert torch.equal(weights[1], clean[1]) and torch.equal(out[1], clean_out[1])
    assert torch.equal(weights[2], old[2]) and not o32[2].any()
    L = lens[0]
    there = np.ones(L, bool)
    for i in gone[0]:
        there[i * 64:i * 64 + 64] = False
    K, V, D = plain.cached(st.kv, st.page_table[0].cpu().numpy(), L)
    lam, q = plain.lam_of(st.stats, 0, st.softmax_scale), plain.tile_rows(st.q4)
    want = np.zeros((H_kv, L))
    for h in range(H_q):
        o, room, top, l = plain.attend(q[0, h], K[h // G], V[h // G], D[h], there[None], lam, 0.5, 8)
        bounded.close(o32[0, h].cpu().numpy(), o[0], room[0], h)
        S = np.where(there, q[0, h, 0] @ K[h // G].T + D[h], -np.inf)
        want[h // G] += np.exp2(lam * (S - top[0])) / l[0]
    close_sums(weights[0, :, :L], old[0, :, :L], want, "present")
    absent = torch.from_numpy(~there).cuda()
    assert torch.equal(weights[0, :, :L][:, absent], old[0, :, :L][:, absent]) and torch.equal(weights[0, :, L:], old[0, :, L:])


# ------------------------------------------------------------------------------------------------------------------ the cache module
def with_spare_pages(st, spare):
    """The same requests in a pool with `spare` more pages; their ids."""
    B = binding()
    n, big = st.kv.num_pages, B.PagedKV.empty(st.kv.num_pages + spare, st.kv.H_q, st.kv.H_kv)
    for new, old in ((big.k_codes, st.kv.k_codes), (big.k_sf, st.kv.k_sf), (big.v_fp8, st.kv.v_fp8), (big.delta, st.kv.delta)):
        new[:n] = old
    st.kv = big
    return torch.arange(n, n + spare, dtype=torch.int32, device="cuda")


def test_a_cache_that_is_cut_back_goes_on_in_a_wider_table():
    """Room for the tokens that follow: more partitions and more logits than the table before had."""
    from paper_2609_33135_b200 import decode_cache
    outs, grown = [], []
    for width in (5, 80):
        st = bounded.state(1540, [900, 300], 8, 2)
        sums = decode_cache.attention_sums(st)
        decode_cache.decode_step(st, weights=sums)
        new_pages = with_spare_pages(st, 2 * width).view(2, width)
        kept, new_sums = decode_cache.evict(st, sums, 300, 4, 100, new_pages)
        assert new_sums.shape == (2, 2, width * 64) and not new_sums[:, :, 300:].any()
        plain_step = decode_cache.decode_step(st).clone()
        assert torch.equal(decode_cache.decode_step(st, window=1 << 20), plain_step)
        assert torch.equal(decode_cache.decode_step(st, weights=new_sums), plain_step)
        again = decode_cache.attention_sums(st)
        decode_cache.decode_step(st, weights=again)
        torch.cuda.synchronize()
        assert int(st.status) == 0
        outs.append(plain_step)
        grown.append(new_sums[:, :, :320])
    assert torch.equal(*outs) and torch.equal(*grown)

@pytest.mark.parametrize("width", [5, 80])   # narrower than the table before, wider
def test_eviction_on_another_stream_than_the_caches(width):
    """What the state gives up is read by calls that have not run yet: other tensors must not get its memory before."""
    from paper_2609_33135_b200 import decode_cache
    sts = [bounded.state(1550, [900, 300], 8, 2) for _ in range(2)]
    kept, outs = [], []
    for k, st in enumerate(sts):
        sums = decode_cache.attention_sums(st)
        decode_cache.decode_step(st, weights=sums)
        new_pages = with_spare_pages(st, 2 * width).view(2, width)
        shapes = [(t.shape, t.dtype) for t in (st.page_table, st.seq_lens, st.workspace)]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            if k:
                torch.cuda._sleep(200_000_000)   # a tenth of a second, so that everything below is asked for before it runs
            kept.append(decode_cache.evict(st, sums, 300, 4, 100, new_pages)[0])
        filled = [torch.full(shape, 1, dtype=dtype, device="cuda") for shape, dtype in shapes for _ in range(64)]
        torch.cuda.synchronize()
        outs.append(decode_cache.decode_step(st).clone())
        assert int(st.status) == 0 and len(filled) == 192
    assert torch.equal(*kept) and torch.equal(*outs)


@pytest.mark.parametrize("width", [5, 80])
def test_a_captured_eviction_keeps_what_it_reads(width):
    """Steps before and after an eviction in one graph, replayed after other tensors have taken all memory that was free."""
    from paper_2609_33135_b200 import decode_cache

    def serve(st, sums, new_pages):
        first = decode_cache.decode_step(st, weights=sums).clone()
        kept, new_sums = decode_cache.evict(st, sums, 300, 4, 100, new_pages)
        return first, kept, new_sums, decode_cache.decode_step(st, weights=new_sums).clone()

    def fresh():
        st = bounded.state(1560, [900, 300], 8, 2)
        return st, decode_cache.attention_sums(st), with_spare_pages(st, 2 * width).view(2, width)

    eager = serve(*fresh())
    torch.cuda.synchronize()
    st, sums, new_pages = fresh()
    shapes = [(t.shape, t.dtype) for t in (st.page_table, st.seq_lens, st.workspace)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = serve(st, sums, new_pages)
    filled = [torch.full(shape, 1, dtype=dtype, device="cuda") for shape, dtype in shapes for _ in range(64)]
    graph.replay()
    torch.cuda.synchronize()
    assert int(st.status) == 0 and len(filled) == 192
    for a, b in zip(eager, captured):
        assert torch.equal(a, b)
def test_sums_leave_the_workspace_of_captured_steps_alone():
    """A graph of a plain step, then sums for the same requests, then the graph again while other tensors take what was given up."""
    from paper_2609_33135_b200 import decode_cache
    st = bounded.state(1570, [2600, 1500], 8, 2)
    decode_cache.decode_step(st)
    want = st.out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode_cache.decode_step(st)
    n = st.workspace.numel()
    sums = decode_cache.attention_sums(st)
    filled = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    st.out.zero_()
    graph.replay()
    decode_cache.decode_step(st, weights=sums)
    torch.cuda.synchronize()
    assert torch.equal(st.out, want) and all(bool((f == 7).all()) for f in filled)


# ------------------------------------------------------------------------------------------------------------------ hidden values
def nan_at(kv, page, t):
    """K scales and Delta_S of one cached token."""
    kv.k_sf[page, :, t * 8:t * 8 + 8] = 0x7F
    for h in range(kv.H_q):
        set_delta(kv, page, h, t, float("nan"))


@pytest.mark.parametrize("lens,q_lens,window,sinks", [
    ([900, 333], None, 100, 5),
    ([1000, 200], [70, 130], 300, 70),
    ([6000], None, 4500, 90),        # accumulated in runs
    ([129, 1], [1, 1], 1, 0),
])
def test_a_chunk_does_not_see_hidden_values_of_pages_that_stay(lens, q_lens, window, sinks):
    """Tokens out of every query's view hold NaN in K and Delta_S; so do those behind the context in its last page."""
    B = binding()
    N_q, nb, H_q, H_kv = 130, len(lens), 8, 2
    st = bounded.state(1580, lens, H_q, H_kv)
    q4 = B.Fp4Tensor.empty(nb, H_q, N_q)
    B.mpfa_quantize_qk(torch.randn(nb, N_q, H_q, 128, generator=torch.Generator().manual_seed(6)).bfloat16().cuda(), None,
                       B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    n = [min(N_q, L) for L in lens] if q_lens is None else q_lens
    n_t = torch.tensor(n, dtype=torch.int32, device="cuda")

    def chunk():
        out, o32 = torch.empty(nb, N_q, H_q, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(nb, N_q, H_q, 128, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.mpfa_prefill_paged_window(q4, st.kv, st.page_table, st.seq_lens, st.stats, 1.0, window, sinks, st.softmax_scale, out, o32, status, n_t)
        assert int(status) == 0
        return o32

    clean, hidden = chunk(), 0
    for b, L in enumerate(lens):
        low = max(L - n[b] - window + 1, 0)
        for i in range(-(-L // 64)):
            for t in range(64):
                if sinks <= i * 64 + t < low or i * 64 + t >= L:
                    nan_at(st.kv, int(st.page_table[b, i]), t)
                    hidden += 1
    assert hidden
    assert torch.equal(chunk(), clean) and bool(clean.any())


@pytest.mark.parametrize("N_q,N_kv,window,sinks", [(130, 900, 100, 5), (200, 1000, 300, 70), (130, 6000, 4500, 90), (1, 333, 1, 0)])
def test_a_prompt_does_not_see_hidden_values(N_q, N_kv, window, sinks):
    """The same on contiguous operands with fewer queries than keys."""
    B = binding()
    w = wl.prefill_workload("hidden", 1590, 2, N_kv, 4, 2, True)
    s1 = B.stage1(w.q[:, :N_q].contiguous().cuda(), w.k.cuda(), w.v.cuda())

    def prompt():
        out, o32 = torch.empty(2, N_q, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, N_q, 4, 128, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.mpfa_prefill_window(s1.q, s1.k, s1.v_fp8, s1.delta, s1.stats, 1.0, window, sinks, w.softmax_scale, out, o32, status)
        assert int(status) == 0
        return o32

    clean = prompt()
    low = max(N_kv - N_q - window + 1, 0)
    pad = -(-N_kv // 128) * 128
    hidden = [j for j in range(pad) if sinks <= j < low or j >= N_kv]
    sf = s1.k.sf.view(-1).view(2, 2, pad // 128, 1024)
    at = [(j // 128, g // 4 * 512 + j % 32 * 16 + j % 128 // 32 * 4 + g % 4) for j in hidden for g in range(8)]
    sf[:, :, [a for a, _ in at], [b for _, b in at]] = 0x7F
    s1.delta.view(2, 4, pad)[:, :, hidden] = float("nan")
    assert hidden and torch.equal(prompt(), clean) and bool(clean.any())


# ------------------------------------------------------------------------------------------------------------------ many and long
def test_weights_of_many_requests():
    """More requests than the kernel holds lengths for, so that work items are found by another rule."""
    lens = [0 if i % 97 == 3 else 1 + (37 * i) % 400 for i in range(780)] + [1500, 2047]
    st = bounded.state(1600, lens, 4, 2)
    old = random_sums(st, 4)
    weights, _, o32, status = sums_of(st, st.page_table, old)
    assert status == 0
    for b, L in enumerate(lens):
        assert torch.equal(weights[b, :, L:], old[b, :, L:])
    for b in (0, 1, 3, 5, 100, 767, 768, 769, 779, 780, 781):
        if lens[b]:
            close_sums(weights[b, :, :lens[b]], old[b, :, :lens[b]], bounded.plain_weights(st, b), b)
        else:
            assert not o32[b].any()


@pytest.mark.parametrize("nb,L,keep", [(1, 20000, 8000), (1, 70000, 9001), (40, 20000, 1000), (75, 49300, 200)])
def test_the_tokens_of_long_rows_arrive(nb, L, keep):
    """Rows of clusters, of one CTA and of more weights than are held: pools of random bytes, every kept token's bytes against those of the slot
    that it comes from, pages that are not the call's left as they were.  Tables share the source pages (they are only read)."""
    H_q, H_kv = 4, 2
    per, pages = -(-keep // 64), -(-L // 64)
    kv, table, spare = bounded.pool(1610 + nb, [L], H_q, H_kv, nb * per)
    table, new_table = table.repeat(nb, 1), spare.view(nb, per)
    lens = [L if b % 3 == 0 else (keep + 1, keep - 1)[b % 2] for b in range(nb)]
    w = torch.rand(nb, H_kv, pages * 64, generator=torch.Generator().manual_seed(nb)).cuda()
    before = bounded.copy_of(kv)
    kept, new_lens, new_weights, status = bounded.evict(kv, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), w, keep, 4, 50, new_table)
    assert status == 0 and new_lens.tolist() == [min(n, keep) for n in lens]
    rest = torch.ones(kv.num_pages, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        rest[new_table[b, :-(-min(n, keep) // 64)].long()] = False
    slot8, half = torch.arange(64, device="cuda") % 8, torch.arange(64, device="cuda") // 8

    def tokens(x):
        """[pages, H_kv, 64, 64 + 8 + 128 + 2 G] bytes of each token, by the maps of mpfa_paged_kv"""
        k = x.k_codes.view(-1, H_kv, 64, 4, 16)
        k = torch.take_along_dim(k, (torch.arange(4, device="cuda") ^ (slot8 // 2)[:, None]).view(1, 1, 64, 4, 1), 3).flatten(3)
        v = x.v_fp8.view(-1, H_kv, 64, 8, 16)
        v = torch.take_along_dim(v, (torch.arange(8, device="cuda") ^ slot8[:, None]).view(1, 1, 64, 8, 1), 3).flatten(3)
        d = x.delta.view(torch.uint8).view(-1, H_kv, H_q // H_kv, 64, 2)
        g = torch.arange(H_q // H_kv, device="cuda")
        d = torch.stack([d[:, :, i][:, :, (half ^ i) * 8 + slot8] for i in g.tolist()], 3).flatten(3)
        return torch.cat((k, x.k_sf.view(-1, H_kv, 64, 8), v, d), 3)

    old, new = tokens(before), tokens(kv)
    assert torch.equal(old[rest], new[rest])
    for b, n in enumerate(lens):
        m = min(n, keep)
        for hk in range(H_kv):
            at = kept[b, hk, :m].long()
            assert bool((at[1:] > at[:-1]).all()) and int(at[0]) >= 0 and int(at[-1]) < n
            rows = new[new_table[b].long(), hk].flatten(0, 1)
            used = -(-m // 64) * 64
            assert torch.equal(rows[:m], old[table[b, at // 64].long(), hk, at % 64]) and not rows[m:used].any()
            assert torch.equal(new_weights[b, hk, :m], w[b, hk, at])
    for b in (0, nb - 1):
        assert np.array_equal(kept[b, 0, :min(lens[b], keep)].cpu().numpy(), plain.evicted(w[b, 0].cpu().numpy(), lens[b], keep, 4, 50))


def test_a_budget_above_what_the_table_holds():
    """Everything is kept, whatever the budget's share of sinks and newest tokens."""
    kv, table, spare = bounded.pool(1620, [300, 5, 0], 8, 2, 3 * 16)
    w, before = torch.rand(3, 2, table.shape[1] * 64, device="cuda"), bounded.copy_of(kv)
    lens, new_table = torch.tensor([300, 5, 0], dtype=torch.int32, device="cuda"), spare.view(3, 16)
    kept, new_lens, new_weights, status = bounded.evict(kv, table, lens, w, 1000, 600, 400, new_table)
    assert status == 0
    bounded.check_evicted(kv, before, table, [300, 5, 0], w, 1000, 600, 400, new_table, kept, new_lens, new_weights)


def test_captured_steps_follow_the_lengths():
    """A step with a window and one with weights, captured once and replayed on lengths from none to all that the table holds."""
    B = binding()
    st = bounded.state(1630, [3000, 3000, 3000], 8, 2)
    table, old = st.page_table, random_sums(st, 7)
    window_out, out, weights = torch.empty_like(st.out), torch.empty_like(st.out), old.clone()
    window_ws = B.decode_window_workspace(3, 8, 2, table.shape[1], 1500, 70)
    ws, status = B.decode_weights_workspace(3, 8, 2, table.shape[1]), torch.zeros(1, dtype=torch.int32, device="cuda")

    def step():
        B.mpfa_decode_window(st.q4, st.kv, table, st.seq_lens, st.stats, 1.0, 1500, 70, st.softmax_scale, window_out, None, window_ws, status)
        B.mpfa_decode_weights(st.q4, st.kv, table, st.seq_lens, st.stats, 1.0, st.softmax_scale, weights, out, None, ws, status)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([0, 0, 0], [1, 3000, 0], [1024, 1025, 64], [2999, 2000, -4], [3000, 3000, 3000]):
        st.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        weights.copy_(old)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        want, want_out, _, _ = sums_of(st, table, old)
        assert torch.equal(weights, want) and torch.equal(out, want_out)
        assert torch.equal(window_out, bounded.window_decode(st, 1500, 70)[0])


@pytest.mark.parametrize("nb,L,keep", [(75, 49300, 4000), (1, 400000, 60000)])   # one CTA to a row; clusters
def test_weights_that_change_during_an_eviction_do_no_harm(nb, L, keep):
    """Which tokens are kept is undefined then; the call ends, and writes nothing beside its buffers."""
    B = binding()
    per, pages = -(-keep // 64), -(-L // 64)
    kv = B.PagedKV.empty(pages + nb * per, 1, 1)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(nb, 1)
    new_table = torch.arange(pages, pages + nb * per, dtype=torch.int32, device="cuda").view(nb, per)
    lens = torch.full((nb,), L, dtype=torch.int32, device="cuda")
    w = torch.rand(nb, 1, pages * 64, device="cuda")
    guard, n = 4096, nb * keep
    arena = torch.full((2 * n + 3 * guard,), -(2 ** 30), dtype=torch.int32, device="cuda")
    kept, new_weights = arena[guard:guard + n].view(nb, 1, keep), arena[2 * guard + n:2 * guard + 2 * n].view(torch.float32).view(nb, 1, keep)
    new_lens, status = torch.empty_like(lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    values = [torch.rand_like(w), torch.rand_like(w) * 1e-6, torch.full_like(w, 0.5)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(100):
        B.mpfa_evict_paged(kv, table, lens, w, keep, 4, 100, new_table, kept, new_lens, new_weights, status)
        with torch.cuda.stream(other):
            for v in values:
                w.copy_(v)
    torch.cuda.synchronize()
    assert int(status) == 0 and new_lens.tolist() == [keep] * nb
    for a, b in ((0, guard), (guard + n, 2 * guard + n), (2 * guard + 2 * n, arena.numel())):
        assert bool((arena[a:b] == -(2 ** 30)).all())
    w.copy_(values[0])   # and with weights that stay, what is always kept
    B.mpfa_evict_paged(kv, table, lens, w, keep, 4, 100, new_table, kept, new_lens, new_weights, status)
    for b in (0, nb - 1):
        assert np.array_equal(kept[b, 0].cpu().numpy(), plain.evicted(w[b, 0].cpu().numpy(), L, keep, 4, 100))


@pytest.mark.parametrize("window,sinks", [(30, 2), (1000, 0), (1, 200)])
def test_a_chunk_longer_than_its_context(window, sinks):
    """Its first queries stand before the first key and see nothing, a whole tile of them among others; one request has no key at all."""
    B = binding()
    lens, N_q, H_q, H_kv = [150, 290, 1, 0], 300, 4, 2
    st = bounded.state(1640, lens, H_q, H_kv)
    q4 = B.Fp4Tensor.empty(4, H_q, N_q)
    B.mpfa_quantize_qk(torch.randn(4, N_q, H_q, 128, generator=torch.Generator().manual_seed(8)).bfloat16().cuda(), None,
                       B.MPFA_SMOOTH | B.MPFA_STATS_FROZEN, st.stats, q4, None, None, None)
    out = torch.full((4, N_q, H_q, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    o32, status = torch.full((4, N_q, H_q, 128), 7.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mpfa_prefill_paged_window(q4, st.kv, st.page_table, st.seq_lens, st.stats, 1.0, window, sinks, st.softmax_scale, out, o32, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    bounded.rounded(out, o32)
    Q = plain.tile_rows(q4)
    for b, L in enumerate(lens):
        got = o32[b].cpu().numpy()
        assert not got[:N_q - L].any()
        if L:
            K, V, D = plain.cached(st.kv, st.page_table[b].cpu().numpy(), L)
            bounded.check_rows(Q[b], K, V, D, got, np.arange(N_q) + L - N_q, window, sinks, plain.lam_of(st.stats, b, st.softmax_scale), 1.0,
                               (H_q, H_kv), b)
