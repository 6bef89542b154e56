"""GPU: the calls for bounded caches where callers, streams and caches are not the plain ones: host threads side by side, pages that are
missing, heads without a softmax, tables that grow, tensors of another stream, hidden values, more requests than the kernels hold lengths for."""
import threading

import numpy as np
import pytest
import torch

import bounded_plain as plain
import test_gpu_bounded as bounded

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
