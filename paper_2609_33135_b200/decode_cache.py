"""Host-side driver for the paged decode path: builds the low-bit KV cache of a
DecodeWorkload by pushing every request through the library's cache-write call, freezes the
query statistics, quantizes the decode-step query and issues mpfa_decode.  All arithmetic is
in the library's kernels; this module only sequences calls and owns the device buffers."""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import List, Optional

import torch

from . import binding as B_
from .workloads import DecodeWorkload


@dataclass
class DecodeState:
    w: DecodeWorkload
    kv: B_.PagedKV
    stats: B_.Stats
    q4: B_.Fp4Tensor
    page_table: torch.Tensor
    seq_lens: torch.Tensor
    workspace: torch.Tensor
    out: torch.Tensor
    out_f32: Optional[torch.Tensor]
    status: torch.Tensor
    v_scale: float
    softmax_scale: float
    sums_workspace: Optional[torch.Tensor] = None   # of steps that sum weights, once there are sums
    captured: List[torch.Tensor] = field(default_factory=list)   # given up during a capture: a replay reads them


def build_cache(w: DecodeWorkload, device="cuda", smooth: bool = True, v_scale: float = 1.0,
                kv_device: str = "cpu", want_f32: bool = True) -> DecodeState:
    """kv_device: where each request's BF16 K/V are drawn ("cpu": same tensors the oracle tests
    use; a CUDA device: drawn in place for the full-size benchmark)."""
    flags = B_.MPFA_SMOOTH if smooth else 0
    stats = B_.Stats.empty(w.B, w.H_q, w.H_kv, device)
    kv = B_.PagedKV.empty(w.num_pages, w.H_q, w.H_kv, with_delta=smooth, device=device)
    ws = B_.quantize_workspace(w.B, w.H_q, w.H_kv, device)
    table = w.page_table.to(device)
    # frozen query statistics from the sample tokens (Section 6: statistics come from prefill)
    qs = w.q_sample.to(device)
    scratch = B_.Fp4Tensor.empty(w.B, w.H_q, qs.shape[1], device)
    B_.mpfa_quantize_qk(qs, None, flags, stats, scratch, None, None, ws)
    for b in range(w.B):
        k, v = w.kv_for_request(b, kv_device)
        k, v = k[0].to(device), v[0].to(device)
        B_.mpfa_quantize_kv_paged(k, v, 0, w.H_q, flags, stats.request(b), v_scale, kv, table[b], ws)
        del k, v
    q4 = B_.Fp4Tensor.empty(w.B, w.H_q, 1, device)
    B_.mpfa_quantize_qk(w.q_new.to(device), None, flags | B_.MPFA_STATS_FROZEN, stats, q4, None, None, None)
    return DecodeState(w, kv, stats, q4, table, w.seq_lens.to(device),
                       B_.decode_workspace(w.B, w.H_q, w.H_kv, table.shape[1], device),
                       torch.empty(w.B, w.H_q, 128, dtype=torch.bfloat16, device=device),
                       torch.empty(w.B, w.H_q, 128, dtype=torch.float32, device=device) if want_f32 else None,
                       torch.zeros(1, dtype=torch.int32, device=device), v_scale, w.softmax_scale)


def decode_step(s: DecodeState, window: Optional[int] = None, sinks: int = 0, weights: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decode step.  window: the query sees the last `window` keys and the first `sinks` only.  weights [B, H_kv, >= 64 * pages]
    (float32): what each key receives of the attention is added to it; of the whole context, so not together with a window."""
    assert window is None or weights is None
    if window is not None:
        B_.mpfa_decode_window(s.q4, s.kv, s.page_table, s.seq_lens, s.stats, s.v_scale, window, sinks, s.softmax_scale, s.out, s.out_f32,
                              s.workspace, s.status)
    elif weights is not None:
        B_.mpfa_decode_weights(s.q4, s.kv, s.page_table, s.seq_lens, s.stats, s.v_scale, s.softmax_scale, weights, s.out, s.out_f32,
                               s.workspace if s.sums_workspace is None else s.sums_workspace, s.status)
    else:
        B_.mpfa_decode(s.q4, s.kv, s.page_table, s.seq_lens, s.stats, s.v_scale, s.softmax_scale, s.out, s.out_f32,
                       s.workspace, s.status)
    return s.out


def _give_up(s: DecodeState, t: torch.Tensor) -> None:
    """Before `s` lets go of a tensor that calls of the current stream may still have to read, which the allocator knows only of the stream that
    it was made on.  A graph that is being captured reads it whenever it is replayed."""
    if not t.is_cuda:
        return
    if torch.cuda.is_current_stream_capturing():
        s.captured.append(t)
    else:
        t.record_stream(torch.cuda.current_stream(t.device))


def _fit_workspaces(s: DecodeState, sums: bool = False) -> None:
    """Larger ones where the page table has outgrown those that are there; with `sums` one for steps that sum weights too."""
    shape, dev = (s.w.B, s.w.H_q, s.w.H_kv, s.page_table.shape[1]), s.page_table.device
    if s.workspace.numel() < B_.lib().mpfa_decode_workspace_bytes(*shape):
        _give_up(s, s.workspace)
        s.workspace = B_.decode_workspace(*shape, dev)
    have = -1 if s.sums_workspace is None else s.sums_workspace.numel()
    if (sums or have >= 0) and have < B_.lib().mpfa_decode_weights_workspace_bytes(*shape):
        if have >= 0:
            _give_up(s, s.sums_workspace)
        s.sums_workspace = B_.decode_weights_workspace(*shape, dev)


def attention_sums(s: DecodeState) -> torch.Tensor:
    """Zeroed sums for decode_step(weights=...), and a workspace for those steps.  The others' stays, since a captured step holds its address."""
    _fit_workspaces(s, sums=True)
    return torch.zeros(s.w.B, s.w.H_kv, s.page_table.shape[1] * B_.PAGE, dtype=torch.float32, device=s.page_table.device)


def evict(s: DecodeState, weights: torch.Tensor, keep: int, sinks: int, recent: int, new_pages: torch.Tensor):
    """Cuts every request's cache back to `keep` tokens a kv head, by `weights`, into the pages of new_pages [B, >= ceil(keep / 64)] (int32; of
    the same pools, in no request's table); from then on `s` has those pages and lengths, and the old pages are the caller's again.
    Returns (the kept tokens' former slots, their sums for further steps: a row is as wide as the new table).
    A graph captured of steps before the eviction has the old table, lengths and workspaces; it is not replayed after it, nor is one with an
    eviction in it once the state is gone."""
    dev = s.page_table.device
    kept = torch.empty(s.w.B, s.w.H_kv, keep, dtype=torch.int32, device=dev)
    new_lens = torch.empty_like(s.seq_lens)
    new_weights = torch.empty(s.w.B, s.w.H_kv, new_pages.shape[1] * B_.PAGE, dtype=torch.float32, device=dev)
    B_.mpfa_evict_paged(s.kv, s.page_table, s.seq_lens, weights, keep, sinks, recent, new_pages, kept, new_lens, new_weights, s.status)
    _give_up(s, s.page_table)
    _give_up(s, s.seq_lens)
    s.page_table, s.seq_lens = new_pages, new_lens
    _fit_workspaces(s)
    return kept, new_weights
