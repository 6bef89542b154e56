"""CPU: what the cache module keeps and replaces for requests whose cache is bounded, and the callables of those calls: what they convert and
refuse."""
import os
import re

import pytest
import torch

from paper_2609_33135_b200 import workloads as wl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def module(monkeypatch):
    """The cache module with the library's calls noted instead of made."""
    from paper_2609_33135_b200 import binding, build, decode_cache
    build.build()
    calls = []
    for name in ("mpfa_decode", "mpfa_decode_window", "mpfa_decode_weights", "mpfa_evict_paged"):
        monkeypatch.setattr(binding, name, lambda *a, name=name: calls.append((name, a)))
    decode_cache.calls = calls
    yield decode_cache
    del decode_cache.calls


def state(module, pages):
    from paper_2609_33135_b200 import binding as B
    w = wl.decode_workload("host", 3, 2, 8, 2, 1, pages * 64, seq_lens=[pages * 64, 5])
    table = torch.zeros(2, pages, dtype=torch.int32)
    return module.DecodeState(w, B.PagedKV.empty(4, 8, 2, device="cpu"), B.Stats.empty(2, 8, 2, "cpu"), None, table, w.seq_lens.clone(),
                              B.decode_workspace(2, 8, 2, pages, "cpu"), torch.empty(2, 8, 128, dtype=torch.bfloat16), None,
                              torch.zeros(1, dtype=torch.int32), 1.0, 0.1)


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_sums_are_fp32_whatever_torchs_default_type(module, default):
    """Programs that build their model in BF16 by setting the default type."""
    st = state(module, 4)
    torch.set_default_dtype(default)
    try:
        sums = module.attention_sums(st)
        _, new_sums = module.evict(st, sums, 100, 4, 10, torch.ones(2, 2, dtype=torch.int32))
    finally:
        torch.set_default_dtype(torch.float32)
    assert sums.dtype == torch.float32 and new_sums.dtype == torch.float32


def test_sums_have_a_workspace_of_their_own(module):
    st = state(module, 20)
    plain = st.workspace
    sums = module.attention_sums(st)
    assert st.workspace is plain and sums.shape == (2, 2, 1280)
    first = st.sums_workspace
    module.attention_sums(st)
    assert st.sums_workspace is first   # large enough still
    module.decode_step(st)
    module.decode_step(st, window=9)
    module.decode_step(st, weights=sums)
    used = {name: a[-2] for name, a in module.calls}   # the workspace stands before the status
    assert used["mpfa_decode"] is plain and used["mpfa_decode_window"] is plain and used["mpfa_decode_weights"] is first


@pytest.mark.parametrize("pages", [2, 20, 21, 500])
def test_workspaces_follow_the_table_after_an_eviction(module, pages):
    from paper_2609_33135_b200 import binding as B
    st = state(module, 20)
    sums = module.attention_sums(st)
    was = st.workspace, st.sums_workspace
    new_pages = torch.ones(2, pages, dtype=torch.int32)
    kept, new_sums = module.evict(st, sums, 100, 4, 10, new_pages)
    assert st.page_table is new_pages and kept.shape == (2, 2, 100) and new_sums.shape == (2, 2, pages * 64)
    L = B.lib()
    assert st.workspace.numel() >= L.mpfa_decode_workspace_bytes(2, 8, 2, pages)
    assert st.sums_workspace.numel() >= L.mpfa_decode_weights_workspace_bytes(2, 8, 2, pages)
    if pages <= 20:
        assert st.workspace is was[0] and st.sums_workspace is was[1]


@pytest.mark.parametrize("call", ["prefill_window", "prefill_paged_window", "decode_window", "decode_weights"])
def test_tensors_that_the_library_would_misread_are_refused(monkeypatch, call):
    """It is given addresses: strides, other types and other sizes go unseen there.  Refused before anything is called."""
    from paper_2609_33135_b200 import binding as B
    n = 1 if call.startswith("decode") else 9
    good = dict(q=B.Fp4Tensor.empty(3, 8, n, "cpu"), kv=B.PagedKV.empty(4, 8, 2, device="cpu"), page_table=torch.zeros(3, 2, dtype=torch.int32),
                seq_lens=torch.ones(3, dtype=torch.int32), stats=B.Stats.empty(3, 8, 2, "cpu"), v_scale=1.0, window=5, sinks=1, softmax_scale=0.1,
                out=torch.empty(3, n, 8, 128, dtype=torch.bfloat16), out_f32=torch.empty(3, n, 8, 128), device_status=torch.zeros(1, dtype=torch.int32))
    strided = torch.ones(3, 2, dtype=torch.int32)[:, 0]
    bad = [{"out": torch.empty(3, n, 8, 128)}, {"out_f32": torch.empty(3, n, 8, 128, dtype=torch.bfloat16)}, {"out": good["out"][:2]},
           {"out": torch.empty(3, n, 8, 256, dtype=torch.bfloat16)[..., :128]}, {"out_f32": torch.empty(3, n, 8, 256)[..., ::2]}]
    if call == "prefill_window":
        for name in ("kv", "page_table", "seq_lens"):
            del good[name]
        good.update(k=B.Fp4Tensor.empty(3, 2, 20, "cpu"), v_fp8=torch.zeros(3 * 2 * 128 * 128, dtype=torch.uint8), delta=None)
    else:
        bad += [{"seq_lens": strided}, {"seq_lens": good["seq_lens"].long()}, {"seq_lens": good["seq_lens"][:2]}, {"page_table": good["page_table"][:2]},
                {"page_table": torch.zeros(2, 3, dtype=torch.int32).T}, {"page_table": good["page_table"].long()}]
        if call == "prefill_paged_window":
            bad += [{"q_lens": strided}, {"q_lens": good["seq_lens"][:2]}]
        else:
            good["workspace"] = torch.empty(1 << 16, dtype=torch.uint8)
        if call == "decode_weights":
            del good["window"], good["sinks"]
            good["weights"] = torch.zeros(3, 2, 128)
            bad += [{"weights": torch.zeros(3, 2, 256)[..., ::2]}, {"weights": torch.zeros(3, 2, 128, dtype=torch.float64)}, {"weights": torch.zeros(2, 2, 128)}]
    made = []
    monkeypatch.setattr(B, "_stream", lambda: made.append(1) or 0)
    monkeypatch.setattr(B, "_check", lambda rc, name: None)
    for change in bad:
        with pytest.raises(AssertionError):
            getattr(B, "mpfa_" + call)(**dict(good, **change))
    assert not made
    larger = {"out": torch.empty(5, n, 8, 128, dtype=torch.bfloat16), "out_f32": None, "seq_lens": torch.ones(7, dtype=torch.int32),
              "page_table": torch.zeros(7, 2, dtype=torch.int32)}   # buffers of a larger batch
    monkeypatch.setattr(B, "lib", lambda: type("Lib", (), {"packed_mpfa_" + call: staticmethod(lambda *a: 0)}))
    getattr(B, "mpfa_" + call)(**dict(good, **{k: v for k, v in larger.items() if k in good}))
    assert made


def entries():
    """name -> kinds of all callables."""
    text = open(os.path.join(ROOT, "paper_2609_33135_b200", "csrc", "calls.c")).read()
    return dict(re.findall(r'^(?:ENTRY|BOUNDED)\((\w+), "(\w+)",', text, flags=re.M))


def test_every_callable_is_found():
    assert len(entries()) == 12


@pytest.mark.parametrize("name", sorted(entries()))
def test_conversions_and_what_is_refused(name):
    from paper_2609_33135_b200 import binding, build
    build.build()
    kinds, call = entries()[name], getattr(binding.lib(), "packed_" + name)
    null = [{"p": None, "i": 1, "f": 1.0, "z": 0}[c] for c in kinds]
    assert call(*null) == -1 and call(*[0 if c == "p" else x for c, x in zip(kinds, null)]) == -1   # None and 0 are null pointers
    for args in (null[:-1], null + [None], []):
        with pytest.raises(TypeError, match="arguments"):
            call(*args)
    bad = {"p": ("text", 1.5, bytearray(8)), "i": (None, 1.5, b"1"), "f": (None, "1"), "z": (None, 1.5)}
    for k, c in enumerate(kinds):
        for x in bad[c]:
            with pytest.raises(TypeError):
                call(*null[:k], x, *null[k + 1:])
        for x in {"i": (1 << 31, -(1 << 31) - 1, 1 << 70), "z": (-1, 1 << 64)}.get(c, ()):
            with pytest.raises(OverflowError):
                call(*null[:k], x, *null[k + 1:])


def test_eviction_bounds_what_changing_weights_could_break():
    """Where a row's weights do not fit shared memory each pass reads them again.  Weights that change between the passes must not make the
    search for the border endless, the list longer than its memory, a row longer than its budget, or a token's slot one that does not exist."""
    from test_launch_rule import bodies, code
    select, move = bodies(code("evict.cu"))["select_tokens"][1], bodies(code("evict.cu"))["evict_move_kernel"][1]
    assert re.search(r"if \(!HELD && by_slot\) break;", select)
    for write in re.findall(r"[^;{}]*(?:sh\.list\[at\] = key|8 \* at, key\)|kept\[at\] = )", select):
        assert re.search(r"HELD \|\| at < (LIST|\(uint32_t\)p\.keep)", write), write
    assert len(re.findall(r"sh\.list\[\w+\] = |, key\);|kept\[[^\]]*\] = ", select)) == 3
    assert re.search(r"min\(\(int\)sh\.listed, LIST\)", select)
    assert 0 < move.index("if (from >= n) from = -1") < move.index("p.weights[head * p.weights_stride + from]")
