"""What the binding of the layer operators refuses (no GPU needed): tensors whose type or layout
the library would read as something else."""
import ctypes

import pytest
import torch

from paper_2609_36246_amd import _lib as L

BF16, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_36246_amd import build
        build.build()
    return L.load()


def qk_args(**change):
    a = dict(positions=torch.zeros(6, dtype=I32), cos=torch.zeros(50, 32), sin=torch.zeros(50, 32),
             weight_q=torch.ones(64, dtype=BF16), weight_k=torch.ones(64, dtype=BF16),
             slots=torch.zeros(6, dtype=I32), slot_rows=9)
    a.update(change)
    return a


def test_a_head_descriptor():
    d = L.make_qk_desc(6, 4, 2, 64, **qk_args())
    assert (d.rot_dim, d.num_positions, d.slot_rows) == (64, 50, 9) and d.positions and d.cos and d.slots
    # fewer rotated elements from tables of their own; none, and tables that are not looked at
    assert L.make_qk_desc(6, 4, 2, 64, **qk_args(cos=torch.zeros(50, 8), sin=torch.zeros(50, 8))).rot_dim == 16
    assert L.make_qk_desc(6, 4, 2, 64, rot_dim=0, **qk_args()).rot_dim == 0
    assert L.make_qk_desc(6, 4, 2, 64, positions=1 << 20, weight_q=1 << 20).positions == 1 << 20


@pytest.mark.parametrize("change", [
    dict(positions=torch.zeros(6, dtype=I64)), dict(positions=torch.zeros(5, dtype=I32)),
    dict(positions=torch.zeros(12, dtype=I32)[::2]), dict(cos=torch.zeros(50, 64)[:, :32]),
    dict(sin=torch.zeros(50, 64)[:, :32]), dict(cos=torch.zeros(50, 32, dtype=BF16)),
    dict(sin=torch.zeros(50, 32, dtype=torch.float64)), dict(sin=torch.zeros(49, 32)),
    dict(sin=torch.zeros(50, 16)), dict(cos=torch.zeros(32, 50).t()), dict(rot_dim=32), dict(num_positions=51),
    dict(weight_q=torch.ones(64)), dict(weight_k=torch.ones(63, dtype=BF16)),
    dict(weight_k=torch.ones(128, dtype=BF16)[::2]), dict(dtype=L.OLIVE_F32), dict(slots=torch.zeros(6, dtype=I64)),
    dict(slots=torch.zeros(5, dtype=I32))], ids=lambda c: "-".join(c))
def test_a_head_descriptor_of_other_arrays(change):
    with pytest.raises(ValueError):
        L.make_qk_desc(6, 4, 2, 64, **qk_args(**change))


def attn_args(**change):
    a = dict(group_seqs=torch.tensor([0, 2, 3], dtype=I32), cu_q=torch.tensor([0, 1, 2, 3], dtype=I32),
             prefix_start=torch.tensor([0, 10]), prefix_len=torch.tensor([10, 5], dtype=I32),
             suffix_len=torch.tensor([1, 2, 3], dtype=I32), suffix_start=torch.tensor([0, 1, 3]), total_q=3, max_q=1,
             max_prefix=10, max_suffix=3, prefix_rows=15, suffix_rows=6)
    a.update(change)
    return a


PAGES = dict(suffix_start=None, page_size=16)


def test_an_attention_descriptor():
    d = L.make_attn_desc(4, 2, 64, **attn_args())
    assert (d.num_groups, d.num_seqs, d.table_stride) == (2, 3, 0)
    table = torch.zeros(4, 9, dtype=I32)[:, 2:5]
    assert L.make_attn_desc(4, 2, 64, **attn_args(page_table=table, **PAGES)).table_stride == 9


@pytest.mark.parametrize("change", [
    dict(group_seqs=torch.tensor([0, 2, 3])), dict(group_seqs=torch.tensor([0, 3], dtype=I32)),
    dict(cu_q=torch.tensor([0, 1, 2, 3])), dict(cu_q=torch.tensor([0, 1, 2], dtype=I32)),
    dict(cu_q=torch.zeros(8, dtype=I32)[::2]), dict(prefix_start=torch.tensor([0, 10], dtype=I32)),
    dict(prefix_len=torch.tensor([10, 5])), dict(suffix_len=torch.tensor([1, 2, 3])),
    dict(suffix_start=torch.tensor([0, 1, 3], dtype=I32)), dict(suffix_start=torch.tensor([0, 1])),
    dict(page_table=torch.zeros(3, 4, dtype=I64), **PAGES), dict(page_table=torch.zeros(2, 4, dtype=I32), **PAGES),
    dict(page_table=torch.zeros(4, 3, dtype=I32).t(), **PAGES), dict(page_table=torch.zeros(12, dtype=I32), **PAGES),
    dict(num_seqs=4)], ids=lambda c: "-".join(c))
def test_an_attention_descriptor_of_other_arrays(change):
    with pytest.raises(ValueError):
        L.make_attn_desc(4, 2, 64, **attn_args(**change))


def test_calls_of_other_tensors(lib, monkeypatch):
    """Heads of another type than the descriptor's, statistics that are not fp32 or too short,
    workspaces with holes: refused before the library is entered."""
    monkeypatch.setattr(L, "_call", lambda name: lambda *a: pytest.fail("the library was entered"))
    h = lambda dtype=BF16: torch.zeros(6, 4, 64, dtype=dtype)  # noqa: E731
    d = L.make_qk_desc(6, 4, 4, 64, weight_q=torch.ones(64, dtype=BF16), weight_k=torch.ones(64, dtype=BF16))
    a = L.make_attn_desc(4, 2, 64, **attn_args())
    bad, gw = [], torch.zeros(64)
    for i in range(4):
        bad.append(lambda i=i: L.olive_qk_norm_rope(d, *[h(F32 if i == j else BF16) for j in range(4)], stream=0))
    for i in range(6):
        bad.append(lambda i=i: L.olive_qk_norm_rope_backward(d, *[h(F32 if i == j else BF16) for j in range(6)],
                                                             stream=0))
        bad.append(lambda i=i: L.olive_prefix_attention(a, *[h(F32 if i == j else BF16) for j in range(6)], stream=0))
    bad += [lambda w=w: L.olive_qk_norm_rope_backward(d, *[h()] * 6, grad_weight_q=w, stream=0)
            for w in (gw.to(BF16), gw[:63], torch.zeros(128)[::2])]
    bad += [lambda s=s: L.olive_prefix_attention(a, *[h()] * 6, lse=s, stream=0)
            for s in (torch.zeros(3, 4, dtype=BF16), torch.zeros(3, 3), torch.zeros(3, 8)[:, ::2])]
    bad += [lambda: L.olive_prefix_attention_backward(a, *[h()] * 6, torch.zeros(3, 3), *[h()] * 6, stream=0),
            lambda: L.olive_prefix_attention(a, *[h()] * 6, workspace=torch.zeros(64)[::2], stream=0),
            lambda: L.olive_grad_clip(1, 1.0, norm=torch.zeros(1, dtype=torch.float64), stream=0)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    # what is an address or a view already is the caller's
    assert isinstance(L.make_heads(h(F32)), L.olive_heads) and ctypes.sizeof(L.olive_heads) == 24


def test_the_current_stream_without_the_bare_handle(monkeypatch):
    """A torch that lacks the entry for a stream's bare handle is asked by its public one."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: type("S", (), {"cuda_stream": 77}))
    assert L._stream(None) == 77 and L._stream(5) == 5
