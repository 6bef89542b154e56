"""CPU: what the calls for bounded caches refuse before any CUDA call, their callables, their workspaces, and the 64-bit statement that the
GPU tests use against the oracle and against a direct count."""
import ctypes
import os
import re

import numpy as np
import pytest

import bounded_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20   # a well-aligned address that nothing dereferences


@pytest.fixture(scope="module")
def binding():
    from paper_2609_33135_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def call(binding, name, good, change):
    args = list(dict(good, **change).values())
    typed, packed = getattr(binding.lib(), name), getattr(binding.lib(), "packed_" + name)
    a = packed(*[bytes(x) if isinstance(x, ctypes.Structure) else x for x in args])
    b = typed(*[ctypes.byref(x) if isinstance(x, ctypes.Structure) else x for x in args])
    assert a == b
    return a


def test_prefill_window_refusals(binding):
    q, k, st = binding._Fp4(A, A, 1, 8, 100), binding._Fp4(A, A, 1, 2, 100), binding._Stats(A, A, A, A)
    good = dict(q=q, k=k, v=A, delta=A, st=st, v_scale=1.0, window=10, sinks=4, scale=0.1, out=A, f32=A, status=A, stream=None)
    nan = float("nan")
    for change, want in (({"window": 0}, -1), ({"window": -1}, -1), ({"sinks": -1}, -1), ({"v": None}, -1), ({"out": None}, -1),
                         ({"status": None}, -1), ({"scale": 0.0}, -1), ({"scale": nan}, -1), ({"v_scale": nan}, -1), ({"v": A + 512}, -3),
                         ({"out": A + 8}, -3), ({"f32": A + 4}, -3), ({"delta": A + 128}, -3),
                         ({"k": binding._Fp4(A, A, 2, 2, 100)}, -1), ({"k": binding._Fp4(A, A, 1, 3, 100)}, -2),
                         ({"q": binding._Fp4(A, A, 1, 18, 100)}, -2), ({"q": binding._Fp4(A + 512, A, 1, 8, 100)}, -3),
                         ({"k": binding._Fp4(A, A, 1, 2, 0)}, -1), ({"q": binding._Fp4(A, A, 1, 8, (1 << 28) + 1)}, -2)):
        assert call(binding, "mpfa_prefill_window", good, change) == want, change


def test_prefill_paged_window_refusals(binding):
    q, kv, st = binding._Fp4(A, A, 2, 8, 100), binding._PagedKV(A, A, A, A, 9, 64, 8, 2), binding._Stats(A, A, A, A)
    good = dict(q=q, kv=kv, table=A, pages=4, lens=A, q_lens=None, st=st, v_scale=1.0, window=10, sinks=4, scale=0.1, out=A, f32=None, status=A,
                stream=None)
    for change, want in (({"window": 0}, -1), ({"sinks": -1}, -1), ({"table": None}, -1), ({"lens": None}, -1), ({"pages": 0}, -1),
                         ({"scale": -1.0}, -1), ({"kv": binding._PagedKV(A, A, A, A, 9, 32, 8, 2)}, -2),
                         ({"kv": binding._PagedKV(A, A, A, A, 9, 64, 6, 2)}, -1), ({"kv": binding._PagedKV(A, A, A, A, 9, 64, 8, 3)}, -2),
                         ({"kv": binding._PagedKV(A, A + 8, A, A, 9, 64, 8, 2)}, -3), ({"out": A + 2}, -3)):
        assert call(binding, "mpfa_prefill_paged_window", good, change) == want, change


def decode_args(binding):
    return dict(q=binding._Fp4(A, A, 3, 8, 1), kv=binding._PagedKV(A, A, A, A, 9, 64, 8, 2), table=A, pages=40, lens=A, st=binding._Stats(A, A, A, A),
                v_scale=1.0)


DECODE = (({"table": None}, -1), ({"lens": None}, -1), ({"pages": 0}, -1), ({"out": None}, -1), ({"ws": None}, -1), ({"status": None}, -1),
          ({"scale": 0.0}, -1), ({"v_scale": -1.0}, -1), ({"nbytes": 0}, -4))


def test_decode_window_refusals(binding):
    n = binding.lib().mpfa_decode_window_workspace_bytes(3, 8, 2, 40, 10, 4)
    good = dict(decode_args(binding), window=10, sinks=4, scale=0.1, out=A, f32=None, ws=A, nbytes=n, status=A, stream=None)
    for change, want in DECODE + (({"window": 0}, -1), ({"window": -5}, -1), ({"sinks": -1}, -1), ({"nbytes": n - 1}, -4), ({"pages": (1 << 24) + 1}, -2),
                                  ({"window": 5000}, -4), ({"q": binding._Fp4(A, A, 3, 8, 2)}, -1), ({"q": binding._Fp4(A, A, 3, 9, 1)}, -1),
                                  ({"kv": binding._PagedKV(A, A, A, A, 9, 64, 8, 3)}, -2), ({"kv": binding._PagedKV(A, A, A + 16, A, 9, 64, 8, 2)}, -3),
                                  ({"ws": A + 8}, -3)):
        assert call(binding, "mpfa_decode_window", good, change) == want, change


def test_decode_weights_refusals(binding):
    n = binding.lib().mpfa_decode_weights_workspace_bytes(3, 8, 2, 40)
    good = dict(decode_args(binding), scale=0.1, weights=A, stride=2560, out=A, f32=None, ws=A, nbytes=n, status=A, stream=None)
    for change, want in DECODE + (({"weights": None}, -1), ({"stride": 2559}, -1), ({"stride": -1}, -1), ({"weights": A + 2}, -3), ({"nbytes": n - 1}, -4),
                                  ({"pages": (1 << 24) + 1}, -2), ({"kv": binding._PagedKV(A, A, A, A, 9, 64, 8, 3)}, -2)):
        assert call(binding, "mpfa_decode_weights", good, change) == want, change


def test_evict_refusals(binding):
    good = dict(kv=binding._PagedKV(A, A, A, A, 9, 64, 8, 2), table=A, B=3, pages=40, lens=A, weights=2 * A, stride=2560, keep=100, sinks=4, recent=20,
                new_table=A, new_pages=2, kept=A, new_lens=A + 64, new_weights=4 * A, new_stride=100, status=A, stream=None)
    for change, want in (({"table": None}, -1), ({"weights": None}, -1), ({"kept": None}, -1), ({"new_weights": None}, -1), ({"new_lens": None}, -1),
                         ({"new_table": None}, -1), ({"status": None}, -1), ({"lens": None}, -1), ({"B": 0}, -1), ({"pages": 0}, -1), ({"keep": 0}, -1),
                         ({"sinks": -1}, -1), ({"recent": -1}, -1), ({"sinks": 60, "recent": 41}, -1), ({"sinks": (1 << 31) - 1, "recent": (1 << 31) - 1}, -1),
                         ({"new_pages": 1}, -1), ({"stride": 2559}, -1), ({"new_stride": 99}, -1),
                         ({"new_weights": 2 * A}, -1), ({"new_weights": 2 * A + 4 * (6 * 2560 - 1)}, -1), ({"weights": 4 * A + 4 * (600 - 1)}, -1),
                         ({"new_lens": A + 8}, -1), ({"kv": binding._PagedKV(A, A, A, A, 9, 32, 8, 2)}, -2),
                         ({"kv": binding._PagedKV(A, A, A, A, 9, 64, 18, 2)}, -2), ({"kv": binding._PagedKV(A, A, A, A, 9, 64, 8, 3)}, -2),
                         ({"kv": binding._PagedKV(A, A, A, A, 0, 64, 8, 2)}, -1), ({"kv": binding._PagedKV(0, A, A, A, 9, 64, 8, 2)}, -1),
                         ({"kv": binding._PagedKV(A + 16, A, A, A, 9, 64, 8, 2)}, -3), ({"weights": 2 * A + 2}, -3), ({"B": 65536}, -2),
                         ({"kept": A + 2}, -3), ({"new_lens": A + 65}, -3), ({"new_table": A + 1}, -3),
                         ({"pages": (1 << 24) + 1}, -2), ({"new_pages": (1 << 24) + 1}, -2)):
        assert call(binding, "mpfa_evict_paged", good, change) == want, change


def test_callables_are_the_declared_argument_types(binding):
    """As for the other entry points: a kind that differs from what is passed, or from the C ABI's type, would go unnoticed."""
    text = open(os.path.join(ROOT, "paper_2609_33135_b200", "csrc", "calls.c")).read()
    found = re.findall(r'^BOUNDED\((\w+), "(\w+)",([^;]*?)\)\n(?=BOUNDED|\n)', text, flags=re.M)
    assert {f[0] for f in found} == {"mpfa_prefill_window", "mpfa_prefill_paged_window", "mpfa_decode_window", "mpfa_decode_weights", "mpfa_evict_paged"}
    letter = {ctypes.c_int: "i", ctypes.c_float: "f", ctypes.c_size_t: "z"}
    for name, kinds, members in found:
        assert kinds == "".join(letter.get(t, "p") for t in getattr(binding.lib(), name).argtypes), name
        assert re.findall(r"v\[(\d+)\]\.(\w)", members) == [(str(k), c) for k, c in enumerate(kinds)], name
        null = [{"p": None, "i": 1, "f": 1.0, "z": 0}[c] for c in kinds]
        packed = getattr(binding.lib(), "packed_" + name)
        assert packed(*null) == -1
        with pytest.raises(TypeError):
            packed(*null[:-1])


def test_windows_need_no_more_partitions_than_the_workspace_holds(binding):
    """The blocks that a window and the sinks reach, counted for every length, against the partition states that the workspace has room for."""
    size = binding.lib().mpfa_decode_window_workspace_bytes
    pages = 80
    for window in (1, 2, 127, 128, 129, 130, 895, 896, 897, 1024, 1025, 3000, 5120, 9000, (1 << 31) - 1):
        for sinks in (0, 1, 128, 129, 1000, 6000, (1 << 31) - 1):
            n = size(1, 1, 1, pages, window, sinks)
            parts = next(p for p in range(1, 20) if (p * 512 + 255) // 256 * 256 + (p * 8 + 255) // 256 * 256 + 256 >= n)
            for L in range(1, pages * 64 + 1, 7):
                j = np.arange(0, L, 1)
                see = (j >= L - window) | (j < sinks)
                blocks = len(np.unique(j[see] // 128))
                assert -(-blocks // 8) <= parts, (window, sinks, L)
    assert size(0, 1, 1, 1, 1, 0) == 0 and size(1, 1, 1, 1, 0, 0) == 0 and size(1, 1, 1, 1, 1, -1) == 0
    assert size(2, 8, 2, 1 << 20, 1024, 4) < 1 << 20   # it follows the window, not the table


def test_the_plain_statement_is_the_oracles():
    """On causal attention and on decode the 64-bit statement and the oracle differ by no more than the statement says they may."""
    from oracle import mpfa_oracle as orc
    from paper_2609_33135_b200 import workloads as wl
    from layouts import codes_to_logical
    assert codes_to_logical is not None
    w = wl.prefill_workload("plain", 7, 1, 300, 4, 2, True, q_bias=True)
    z = orc.stage1(orc.bf16_bits(w.q), orc.bf16_bits(w.k), orc.bf16_bits(w.v), v_scale=0.5)
    Q = plain.e2m1(z.q_codes) * np.repeat(plain.E4M3[z.q_sf], 16, -1)
    K = plain.e2m1(z.k_codes) * np.repeat(plain.E4M3[z.k_sf], 16, -1)
    V = plain.E4M3[z.v_codes]
    D = (z.delta.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    lam = w.softmax_scale / np.log(2.0) * float(z.dq[0]) * float(z.dk[0])
    rows = orc.all_rows(1, 4, 300)
    ref, _ = orc.prefill_rows(z, rows, w.softmax_scale, True)
    got = {(h, i): x for (_, h, i), x in zip(rows, ref)}
    for h in range(4):
        for r in range(0, 300, 128):
            pos = np.arange(r, min(r + 128, 300))
            want, room, _, _ = plain.attend(Q[0, h, pos], K[0, h // 2, :300], V[0, h // 2, :300], D[0, h, :300], plain.visible(pos, 300, 300, 0), lam, 0.5, 0)
            assert (np.abs(np.stack([got[h, i] for i in pos]) - want) <= room).all()


def test_the_launch_rule_covers_the_kernels():
    from test_launch_rule import launched
    assert {"decode_weights_kernel", "evict_select_kernel", "evict_move_kernel"} <= launched()


def test_the_plain_visibility_by_hand():
    assert plain.visible([5], 8, 2, 1).astype(int).tolist() == [[1, 0, 0, 0, 1, 1, 0, 0]]
    assert plain.visible([0, -1], 2, 1, 2).astype(int).tolist() == [[1, 0], [0, 0]]
    see = plain.visible(range(640, 700), 700, 100, 3)
    assert plain.lists_of_blocks(see, 0) == [[0, 4, 5]] and plain.lists_of_blocks(see, 2) == [[0, 4], [5]]
    w = np.array([3, 1, 2, 2, 5, np.nan, 0], np.float32)
    assert plain.evicted(w, 7, 4, 1, 1).tolist() == [0, 2, 4, 6] and plain.evicted(w, 7, 3, 0, 0).tolist() == [0, 2, 4]
