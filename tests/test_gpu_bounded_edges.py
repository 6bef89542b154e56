"""GPU: the calls for bounded caches where callers, streams and caches are not the plain ones: host threads side by side, pages that are
missing, heads without a softmax, tables that grow, tensors of another stream, hidden values, more requests than the kernels hold lengths for."""
import threading

import numpy as np
import pytest
import torch

import bounded_plain as plain

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
