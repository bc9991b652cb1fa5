"""Host-side checks of include/olive_layers.h (no GPU needed): the library exports what the
header declares, the binding's structs and constants are the header's, and malformed
arguments are rejected before the device is touched."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_36246_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "olive_layers.h")
P = 1 << 20                                   # an address that is never followed
STRUCTS = ("olive_heads", "olive_qk_desc", "olive_attn_desc", "olive_grad_tensor")


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_36246_amd import build
        build.build()
    return L.load()


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_exports(lib):
    names = set(re.findall(r"\b(olive_[a-z_]+)\s*\(", text()))
    assert names == {"olive_qk_norm_rope", "olive_qk_norm_rope_workspace", "olive_qk_norm_rope_backward",
                     "olive_prefix_attention", "olive_prefix_attention_workspace",
                     "olive_prefix_attention_backward", "olive_grad_clip_init", "olive_grad_clip",
                     "olive_grad_clip_free"}
    for n in names:
        assert hasattr(lib, n) and hasattr(L, n), n


def test_constants():
    defs = re.findall(r"^#define\s+(OLIVE_[A-Z0-9_]+)\s+(\d+)", open(HEADER).read(), re.M)
    assert len(defs) == 2
    for name, value in defs:
        assert getattr(L, name) == int(value)


def test_struct_layouts(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "olive_layers.h"', "int main(void) {"]
    for name in STRUCTS:
        lines.append('printf("%s . %%zu\\n", sizeof(%s));' % (name, name))
        for f, _ in getattr(L, name)._fields_:
            lines.append('printf("%s %s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f))
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0;", "}"]) + "\n")
    subprocess.run([cc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o",
                    str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout
    for line in out.splitlines():
        name, field, value = line.split()
        st = getattr(L, name)
        assert int(value) == (ctypes.sizeof(st) if field == "." else getattr(st, field).offset), line


def view(p=P, st=256, sh=64):
    return L.olive_heads(p, st, sh)


def set_fields(d, change):
    for k, v in change.items():
        setattr(d, k, v)
    return d


def qk_desc(**change):
    d = L.make_qk_desc(8, 4, 2, 64, positions=P, cos=None, sin=None, weight_q=P, weight_k=P)
    d.rot_dim, d.num_positions, d.cos, d.sin = 64, 100, P, P
    return set_fields(d, change)


E = L
QK_BAD = [("size", 8, E.OLIVE_E_RANGE), ("dtype", 2, E.OLIVE_E_DTYPE), ("tokens", -1, E.OLIVE_E_SHAPE),
          ("tokens", 1 << 31, E.OLIVE_E_SHAPE), ("heads_q", -1, E.OLIVE_E_SHAPE),
          ("heads_k", 5000, E.OLIVE_E_UNSUPPORTED), ("head_dim", 0, E.OLIVE_E_SHAPE),
          ("head_dim", 257, E.OLIVE_E_UNSUPPORTED), ("rot_dim", 63, E.OLIVE_E_RANGE),
          ("rot_dim", 66, E.OLIVE_E_RANGE), ("rot_dim", -2, E.OLIVE_E_RANGE), ("layout", 2, E.OLIVE_E_RANGE),
          ("eps", float("nan"), E.OLIVE_E_RANGE), ("eps", -1.0, E.OLIVE_E_RANGE),
          ("positions", None, E.OLIVE_E_NULL), ("cos", None, E.OLIVE_E_NULL),
          ("num_positions", 0, E.OLIVE_E_SHAPE)]


@pytest.mark.parametrize("field,value,status", QK_BAD)
def test_qk_descriptor(field, value, status):
    d, h = qk_desc(**{field: value}), view()
    assert L.olive_qk_norm_rope(d, h, h, h, h, stream=0, check=False) == status
    assert L.olive_qk_norm_rope_backward(d, h, h, h, h, h, h, stream=0, check=False) == status
    with pytest.raises(L.OliveError) as e:
        L.olive_qk_norm_rope_workspace(d)
    assert e.value.status == status


def test_qk_views():
    d, h, none = qk_desc(), view(), view(None)
    call = lambda *a, **k: L.olive_qk_norm_rope(d, *a, stream=0, check=False, **k)  # noqa: E731
    assert call(None, h, h, h) == E.OLIVE_E_NULL
    assert call(h, h, h, none) == E.OLIVE_E_NULL
    assert call(h, h, h, h, v=h) == E.OLIVE_E_NULL
    assert call(view(P + 1), h, h, h) == E.OLIVE_E_UNSUPPORTED
    d.heads_q = d.heads_k = 0
    assert call(h, h, h, h) == E.OLIVE_E_SHAPE
    assert L.olive_qk_norm_rope(qk_desc(tokens=0), h, h, h, h, stream=0, check=False) == E.OLIVE_OK
    assert L.load().olive_qk_norm_rope(None, h, h, h, h, h, h, None) == E.OLIVE_E_NULL


def test_qk_backward_workspace():
    d, h = qk_desc(), ctypes.byref(view())
    need = L.olive_qk_norm_rope_workspace(d)
    assert need > 0

    def call(d, gwq, gwk, work, n):
        return L.load().olive_qk_norm_rope_backward(ctypes.byref(d), h, h, h, h, h, h, gwq, gwk, work, n, None)

    assert call(d, P, P, None, need) == E.OLIVE_E_NULL
    assert call(d, P, None, P, need - 1) == E.OLIVE_E_SHAPE
    assert call(d, None, P, P + 8, need) == E.OLIVE_E_UNSUPPORTED
    assert call(qk_desc(weight_q=None), P, P, P, need) == E.OLIVE_E_NULL


def attn_desc(page=False, **change):
    d = L.make_attn_desc(4, 2, 64, P, P, P, P, P, total_q=40, max_q=20, max_prefix=100, max_suffix=50,
                         prefix_rows=200, suffix_rows=320, suffix_start=None if page else P,
                         page_table=P if page else None, page_size=16 if page else 0, num_groups=2, num_seqs=4)
    if page:
        d.table_stride = 4
    return set_fields(d, change)


ATTN_BAD = [("size", 0, E.OLIVE_E_RANGE), ("dtype", -1, E.OLIVE_E_DTYPE), ("num_groups", 0, E.OLIVE_E_SHAPE),
            ("num_groups", 5, E.OLIVE_E_SHAPE), ("num_seqs", 1 << 20, E.OLIVE_E_SHAPE),
            ("heads_kv", 0, E.OLIVE_E_SHAPE), ("heads_kv", 3, E.OLIVE_E_SHAPE),
            ("heads_q", 1, E.OLIVE_E_SHAPE), ("head_dim", 0, E.OLIVE_E_SHAPE),
            ("head_dim", 257, E.OLIVE_E_UNSUPPORTED), ("max_q", 0, E.OLIVE_E_SHAPE),
            ("total_q", -1, E.OLIVE_E_SHAPE), ("max_prefix", -1, E.OLIVE_E_SHAPE),
            ("max_suffix", 1 << 31, E.OLIVE_E_SHAPE), ("prefix_rows", -1, E.OLIVE_E_SHAPE),
            ("scale", float("inf"), E.OLIVE_E_RANGE), ("group_seqs", None, E.OLIVE_E_NULL),
            ("cu_q", None, E.OLIVE_E_NULL), ("suffix_len", None, E.OLIVE_E_NULL),
            ("suffix_start", None, E.OLIVE_E_NULL), ("page_table", P, E.OLIVE_E_NULL)]


def attn_forward(d, views=None, lse=None, work=P, size=1 << 40):
    v = [ctypes.byref(view())] * 6 if views is None else views
    return L.load().olive_prefix_attention(ctypes.byref(d), *v, lse, work, size, None)


def attn_backward(d, work=P, size=1 << 40, lse=P):
    v = [ctypes.byref(view())] * 6
    return L.load().olive_prefix_attention_backward(ctypes.byref(d), *v, lse, *v, work, size, None)


@pytest.mark.parametrize("field,value,status", ATTN_BAD)
def test_attention_descriptor(field, value, status):
    d = attn_desc(**{field: value})
    assert attn_forward(d) == status and attn_backward(d) == status
    n = ctypes.c_int64()
    assert L.load().olive_prefix_attention_workspace(ctypes.byref(d), 0, ctypes.byref(n)) == status


def test_attention_pages_and_views():
    assert attn_forward(attn_desc(page=True, table_stride=3)) == E.OLIVE_E_SHAPE
    assert attn_forward(attn_desc(page=True, page_size=0)) == E.OLIVE_E_SHAPE
    assert attn_backward(attn_desc(page=True)) == E.OLIVE_E_UNSUPPORTED
    h = ctypes.byref(view())
    assert attn_forward(attn_desc(), [None] + [h] * 5) == E.OLIVE_E_NULL
    assert attn_forward(attn_desc(), [h, None] + [h] * 4) == E.OLIVE_E_NULL
    assert attn_forward(attn_desc(), [h] * 4 + [None, h]) == E.OLIVE_E_NULL
    assert attn_forward(attn_desc(), [h] * 5 + [ctypes.byref(view(P + 1))]) == E.OLIVE_E_UNSUPPORTED
    assert attn_backward(attn_desc(), lse=None) == E.OLIVE_E_NULL
    assert attn_forward(attn_desc(total_q=0)) == E.OLIVE_OK


def test_attention_workspace():
    d = attn_desc()
    n = [ctypes.c_int64(), ctypes.c_int64()]
    for i in (0, 1):
        assert L.load().olive_prefix_attention_workspace(ctypes.byref(d), i, ctypes.byref(n[i])) == E.OLIVE_OK
    assert L.olive_prefix_attention_workspace(d) == n[0].value
    assert L.olive_prefix_attention_workspace(d, backward=True) == max(n[0].value, n[1].value)
    need = n[1].value
    assert attn_backward(d, size=need - 1) == E.OLIVE_E_SHAPE
    assert attn_backward(d, work=None) == E.OLIVE_E_NULL
    assert attn_backward(d, work=P + 4) == E.OLIVE_E_UNSUPPORTED
    long = L.make_attn_desc(16, 8, 128, P, P, P, P, P, total_q=4, max_q=1, max_prefix=1 << 17,
                            max_suffix=1024, prefix_rows=1 << 17, suffix_rows=4096, suffix_start=P,
                            num_groups=1, num_seqs=4)
    need = L.olive_prefix_attention_workspace(long)
    if need:
        assert attn_forward(long, size=need - 1) == E.OLIVE_E_SHAPE
        assert attn_forward(long, work=None) == E.OLIVE_E_NULL


def test_clip_arguments():
    init = L.load().olive_grad_clip_init
    h = ctypes.c_void_p()

    def status(count=1, out=ctypes.byref(h), **change):
        t = set_fields(L.olive_grad_tensor(P, P, 10, L.OLIVE_F32, L.OLIVE_F32), change)
        return init(out, ctypes.byref(t), count, None)

    assert status(out=None) == E.OLIVE_E_NULL
    assert init(ctypes.byref(h), None, 1, None) == E.OLIVE_E_NULL
    assert status(count=-1) == E.OLIVE_E_SHAPE
    assert status(n=-1) == E.OLIVE_E_SHAPE
    assert status(grad=None) == E.OLIVE_E_NULL
    assert status(dtype=9) == E.OLIVE_E_DTYPE
    assert status(dtype_out=9) == E.OLIVE_E_DTYPE
    assert status(dtype_out=L.OLIVE_BF16) == E.OLIVE_E_RANGE
    assert status(grad=P + 2) == E.OLIVE_E_UNSUPPORTED
    assert status(n=1 << 62) in (E.OLIVE_E_SHAPE, E.OLIVE_E_NOMEM)
    assert h.value is None
    assert L.olive_grad_clip(None, 1.0, stream=0, check=False) == E.OLIVE_E_NULL
    assert L.olive_grad_clip_free(None) == E.OLIVE_OK


def test_binding_checks_views():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        L.make_heads(torch.zeros(4, 8))
    with pytest.raises(ValueError):
        L.make_heads(torch.zeros(4, 8, 16).transpose(1, 2))
    h = L.make_heads(torch.zeros(4, 8, 16)[:, 2:5])
    assert (h.stride_token, h.stride_head) == (128, 16)
    with pytest.raises(ValueError):
        L.olive_grad_clip_init([torch.zeros(4, 8).t()])
    with pytest.raises(ValueError):
        L.olive_grad_clip_init([torch.zeros(4)], [torch.zeros(3)])
    with pytest.raises(ValueError):
        L.olive_grad_clip_init([torch.zeros(4)], [])
