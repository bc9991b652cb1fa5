"""Host-side checks of include/olive_tokens.h (no GPU needed): the library exports what the
header declares, the binding's structs and constants are the header's, malformed arguments are
rejected before the device is touched, and the binding refuses tensors that the library would
read as something else."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2609_36246_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "olive_tokens.h")
P = 1 << 20                                   # an address that is never followed
BF16, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
STRUCTS = ("olive_embed_desc", "olive_norm_desc", "olive_sample_desc")
E = L


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
    assert names == {"olive_embed", "olive_embed_workspace", "olive_embed_backward", "olive_row_norm",
                     "olive_row_norm_workspace", "olive_row_norm_backward", "olive_sample_workspace", "olive_sample"}
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
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "olive_tokens.h"', "int main(void) {"]
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


def set_fields(d, change):
    for k, v in change.items():
        setattr(d, k, v)
    return d


def refused(desc, calls, status):
    for call in calls:
        assert call(desc) == status
    n = ctypes.c_int64()
    name = {L.olive_embed_desc: "olive_embed", L.olive_norm_desc: "olive_row_norm", L.olive_sample_desc: "olive_sample"}
    assert getattr(L.load(), name[type(desc)] + "_workspace")(ctypes.byref(desc), ctypes.byref(n)) == status
    with pytest.raises(L.OliveError) as e:
        L._bytes_of(name[type(desc)] + "_workspace", desc)
    assert e.value.status == status


# ----------------------------------------------------------------------------- embedding
def embed_desc(**change):
    return set_fields(L.make_embed_desc(8, 100, 64, P), change)


def embed(d, table=P, ts=64, out=P, os_=64):
    return L.load().olive_embed(ctypes.byref(d), table, ts, out, os_, None)


def embed_backward(d, grad=P, gs=64, table=P, ts=64, kind=0, add=0, work=P, size=1 << 40):
    return L.load().olive_embed_backward(ctypes.byref(d), grad, gs, table, ts, kind, add, work, size, None)


@pytest.mark.parametrize("field,value,status", [
    ("size", 0, E.OLIVE_E_RANGE), ("dtype", 2, E.OLIVE_E_DTYPE), ("tokens", -1, E.OLIVE_E_SHAPE),
    ("tokens", (1 << 26) + 1, E.OLIVE_E_UNSUPPORTED), ("vocab", 0, E.OLIVE_E_SHAPE), ("vocab", 1 << 31, E.OLIVE_E_SHAPE),
    ("width", 0, E.OLIVE_E_SHAPE), ("width", 65537, E.OLIVE_E_UNSUPPORTED), ("scale", float("inf"), E.OLIVE_E_RANGE),
    ("scale", float("nan"), E.OLIVE_E_RANGE), ("ids", None, E.OLIVE_E_NULL)])
def test_embed_descriptor(field, value, status):
    refused(embed_desc(**{field: value}), (embed, embed_backward), status)


def test_embed_matrices():
    d = embed_desc()
    assert embed(d, table=None) == E.OLIVE_E_NULL and embed(d, out=None) == E.OLIVE_E_NULL
    assert embed(d, os_=63) == E.OLIVE_E_SHAPE and embed(d, ts=-1) == E.OLIVE_E_SHAPE
    assert embed(d, ts=1 << 60) == E.OLIVE_E_SHAPE and embed(d, os_=1 << 59) == E.OLIVE_E_SHAPE
    assert embed(d, table=P + 1) == E.OLIVE_E_UNSUPPORTED and embed(d, out=P + 1) == E.OLIVE_E_UNSUPPORTED
    assert embed(embed_desc(tokens=0, ids=None), None, 0, None, 0) == E.OLIVE_OK
    assert L.load().olive_embed(None, P, 64, P, 64, None) == E.OLIVE_E_NULL
    assert embed_backward(d, grad=None) == E.OLIVE_E_NULL and embed_backward(d, table=None) == E.OLIVE_E_NULL
    assert embed_backward(d, gs=-1) == E.OLIVE_E_SHAPE and embed_backward(d, ts=63) == E.OLIVE_E_SHAPE
    assert embed_backward(d, ts=0) == E.OLIVE_E_SHAPE
    assert embed_backward(d, kind=2) == E.OLIVE_E_DTYPE and embed_backward(d, add=2) == E.OLIVE_E_RANGE
    assert embed_backward(d, table=P + 2) == E.OLIVE_E_UNSUPPORTED
    assert embed_backward(d, grad=P + 1) == E.OLIVE_E_UNSUPPORTED
    assert embed_backward(embed_desc(tokens=0, ids=None), None, 0, P, 64, add=1) == E.OLIVE_OK


def test_embed_workspace():
    for n in (0, 1, 8, 3000, 40000, 1 << 20, 1 << 26):
        d = embed_desc(tokens=n)
        need = L.olive_embed_workspace(d)
        assert need >= 0
        if need:
            assert embed_backward(d, size=need - 1) == E.OLIVE_E_SHAPE
            assert embed_backward(d, work=None) == E.OLIVE_E_NULL
            assert embed_backward(d, work=P + 8) == E.OLIVE_E_UNSUPPORTED
    assert L.load().olive_embed_workspace(ctypes.byref(embed_desc()), None) == E.OLIVE_E_NULL


# ----------------------------------------------------------------------------- row norms
def norm_desc(**change):
    return set_fields(L.make_norm_desc(8, 64, P, P), change)


def norm(d, x=P, xs=64, res=None, rs=0, out=P, os_=64, total=None, ts=0):
    return L.load().olive_row_norm(ctypes.byref(d), x, xs, res, rs, out, os_, total, ts, None)


def norm_backward(d, h=P, hs=64, g=P, gs=64, s=None, ss=0, gh=P, ghs=64, gw=None, gb=None, work=P, size=1 << 40):
    return L.load().olive_row_norm_backward(ctypes.byref(d), h, hs, g, gs, s, ss, gh, ghs, gw, gb, work, size, None)


@pytest.mark.parametrize("field,value,status", [
    ("size", 8, E.OLIVE_E_RANGE), ("dtype", -1, E.OLIVE_E_DTYPE), ("rows", -1, E.OLIVE_E_SHAPE),
    ("rows", 1 << 31, E.OLIVE_E_SHAPE), ("width", 0, E.OLIVE_E_SHAPE), ("width", 16385, E.OLIVE_E_UNSUPPORTED),
    ("kind", 2, E.OLIVE_E_RANGE), ("eps", -1e-6, E.OLIVE_E_RANGE), ("eps", float("nan"), E.OLIVE_E_RANGE),
    ("weight", P + 1, E.OLIVE_E_UNSUPPORTED), ("bias", P + 1, E.OLIVE_E_UNSUPPORTED)])
def test_norm_descriptor(field, value, status):
    refused(norm_desc(**{field: value}), (norm, norm_backward), status)


def test_norm_matrices():
    d = norm_desc()
    assert norm(d, x=None) == E.OLIVE_E_NULL and norm(d, out=None) == E.OLIVE_E_NULL
    assert norm(d, xs=-1) == E.OLIVE_E_SHAPE and norm(d, os_=63) == E.OLIVE_E_SHAPE
    assert norm(d, res=P, rs=-5) == E.OLIVE_E_SHAPE and norm(d, total=P, ts=0) == E.OLIVE_E_SHAPE
    for k in ("x", "res", "out", "total"):
        assert norm(d, **{k: P + 1, "rs": 64, "ts": 64}) == E.OLIVE_E_UNSUPPORTED
    assert norm(norm_desc(rows=0), None, 0, None, 0, None, 0) == E.OLIVE_OK
    assert L.load().olive_row_norm(None, P, 64, None, 0, P, 64, None, 0, None) == E.OLIVE_E_NULL
    for k in ("h", "g", "gh"):
        assert norm_backward(d, **{k: None}) == E.OLIVE_E_NULL
        assert norm_backward(d, **{k: P + 1}) == E.OLIVE_E_UNSUPPORTED
    assert norm_backward(d, ghs=0) == E.OLIVE_E_SHAPE and norm_backward(d, s=P, ss=-1) == E.OLIVE_E_SHAPE
    assert norm_backward(d, gw=P + 2) == E.OLIVE_E_UNSUPPORTED and norm_backward(d, gb=P + 1) == E.OLIVE_E_UNSUPPORTED
    need = L.olive_row_norm_workspace(d)
    assert need > 0
    assert norm_backward(d, gw=P, size=need - 1) == E.OLIVE_E_SHAPE
    assert norm_backward(d, gb=P, work=None) == E.OLIVE_E_NULL
    assert norm_backward(d, gb=P, work=P + 4) == E.OLIVE_E_UNSUPPORTED
    assert norm_backward(norm_desc(rows=0), None, 0, None, 0, None, 0, None, 0, work=None, size=0) == E.OLIVE_OK
    assert L.load().olive_row_norm_workspace(ctypes.byref(d), None) == E.OLIVE_E_NULL


# ------------------------------------------------------------------------------ sampling
def sample_desc(**change):
    return set_fields(L.make_sample_desc(8, 100, P), change)


def sample(d, logits=P, stride=100, token=P, logp=None, kept=None, work=P, size=1 << 40):
    return L.load().olive_sample(ctypes.byref(d), logits, stride, token, logp, kept, work, size, None)


@pytest.mark.parametrize("field,value,status", [
    ("size", 8, E.OLIVE_E_RANGE), ("dtype", 5, E.OLIVE_E_DTYPE), ("rows", -1, E.OLIVE_E_SHAPE),
    ("rows", (1 << 20) + 1, E.OLIVE_E_UNSUPPORTED), ("vocab", 0, E.OLIVE_E_SHAPE),
    ("vocab", (1 << 24) + 1, E.OLIVE_E_UNSUPPORTED), ("uniform", None, E.OLIVE_E_NULL)])
def test_sample_descriptor(field, value, status):
    refused(sample_desc(**{field: value}), (sample,), status)


def test_sample_arguments():
    d = sample_desc()
    assert sample(d, logits=None) == E.OLIVE_E_NULL and sample(d, token=None) == E.OLIVE_E_NULL
    assert sample(d, stride=-1) == E.OLIVE_E_SHAPE and sample(d, stride=1 << 60) == E.OLIVE_E_SHAPE
    assert sample(d, logits=P + 1) == E.OLIVE_E_UNSUPPORTED
    assert sample(sample_desc(rows=0, uniform=None), None, 0, None) == E.OLIVE_OK
    assert L.load().olive_sample(None, P, 100, P, None, None, P, 1 << 40, None) == E.OLIVE_E_NULL
    assert L.load().olive_sample_workspace(ctypes.byref(d), None) == E.OLIVE_E_NULL
    for rows, vocab in ((1, 1), (1, 151936), (64, 151936), (2048, 32000), (1 << 20, 1 << 24)):
        for dtype in (L.OLIVE_BF16, L.OLIVE_F32):
            d = sample_desc(rows=rows, vocab=vocab, dtype=dtype)
            need = L.olive_sample_workspace(d)
            if need:
                assert sample(d, stride=vocab, size=need - 1) == E.OLIVE_E_SHAPE
                assert sample(d, stride=vocab, work=None) == E.OLIVE_E_NULL
                assert sample(d, stride=vocab, work=P + 8) == E.OLIVE_E_UNSUPPORTED


# --------------------------------------------------------------------------- the binding
def test_calls_of_other_tensors(monkeypatch):
    """Matrices of another type, size or layout, overlapping output rows: refused before the
    library is entered."""
    monkeypatch.setattr(L, "_call", lambda name: lambda *a: pytest.fail("the library was entered"))
    m = lambda n=6, w=64, dtype=BF16: torch.zeros(n, w, dtype=dtype)  # noqa: E731
    others = lambda n=6, dtype=BF16: [m(n, dtype=F32 if dtype is BF16 else BF16), m(n + 1, dtype=dtype),  # noqa: E731
                                      m(n, 63, dtype), m(64, n, dtype).t(), m(n, 128, dtype)[:, ::2], m(n * 64, 1, dtype)]
    ids = torch.zeros(6, dtype=I32)
    e, k = L.make_embed_desc(6, 9, 64, ids), L.make_norm_desc(6, 64)
    s = L.make_sample_desc(6, 64, torch.zeros(6))
    one = torch.zeros(1, 64, dtype=BF16).expand(6, 64)
    tok = torch.zeros(6, dtype=I32)
    bad = [lambda t=t: L.olive_embed(e, t, m(), stream=0) for t in others(9)]
    bad += [lambda t=t: L.olive_embed(e, m(9), t, stream=0) for t in others() + [one]]
    bad += [lambda t=t: L.olive_embed_backward(e, t, m(9, dtype=F32), stream=0) for t in others()]
    bad += [lambda t=t: L.olive_embed_backward(e, m(), t, stream=0) for t in others(9, F32)[1:] + [m(9, dtype=torch.float64)]]
    bad += [lambda t=t: L.olive_embed_backward(e, m(), t, stream=0) for t in (m(1, dtype=F32).expand(9, 64),)]
    bad += [lambda: L.olive_embed_backward(e, m(), m(9), workspace=torch.zeros(64)[::2], stream=0)]
    for t in others():
        bad += [lambda t=t: L.olive_row_norm(k, t, m(), stream=0), lambda t=t: L.olive_row_norm(k, m(), t, stream=0),
                lambda t=t: L.olive_row_norm(k, m(), m(), residual=t, stream=0),
                lambda t=t: L.olive_row_norm(k, m(), m(), sum_out=t, stream=0),
                lambda t=t: L.olive_row_norm_backward(k, t, m(), m(), stream=0),
                lambda t=t: L.olive_row_norm_backward(k, m(), t, m(), stream=0),
                lambda t=t: L.olive_row_norm_backward(k, m(), m(), t, stream=0),
                lambda t=t: L.olive_row_norm_backward(k, m(), m(), m(), grad_sum=t, stream=0),
                lambda t=t: L.olive_sample(s, t, tok, stream=0)]
    bad += [lambda: L.olive_row_norm(k, m(), one, stream=0), lambda: L.olive_row_norm(k, m(), m(), sum_out=one, stream=0),
            lambda: L.olive_row_norm_backward(k, m(), m(), one, stream=0)]
    bad += [lambda w=w: L.olive_row_norm_backward(k, m(), m(), m(), grad_weight=w, stream=0)
            for w in (torch.zeros(63), torch.zeros(64, dtype=BF16), torch.zeros(128)[::2])]
    bad += [lambda t=t: L.olive_sample(s, m(), t, stream=0) for t in (tok.long(), tok[:5], torch.zeros(12, dtype=I32)[::2])]
    bad += [lambda: L.olive_sample(s, m(), tok, logp=torch.zeros(6, dtype=torch.float64), stream=0),
            lambda: L.olive_sample(s, m(), tok, kept=torch.zeros(6), stream=0)]
    for call in bad:
        with pytest.raises(ValueError, match="expected|contiguous"):
            call()


def test_tensors_of_another_device(monkeypatch):
    """What is not on the current device is refused before the library is entered."""
    monkeypatch.setattr(L, "_call", lambda name: lambda *a: pytest.fail("the library was entered"))
    monkeypatch.setattr(L, "_here", lambda: 3)
    x, ids, f = torch.zeros(6, 64, dtype=BF16), torch.zeros(6, dtype=I32), torch.zeros(6)
    e, k, s = L.make_embed_desc(6, 6, 64, ids), L.make_norm_desc(6, 64), L.make_sample_desc(6, 64, f)
    for call in (lambda: L.olive_embed(e, x, x, stream=0), lambda: L.olive_embed_backward(e, x, x, stream=0),
                 lambda: L.olive_row_norm(k, x, x, stream=0), lambda: L.olive_row_norm_backward(k, x, x, x, stream=0),
                 lambda: L.olive_sample(s, x, ids, stream=0)):
        with pytest.raises(ValueError, match="on device -1, and the current one is 3"):
            call()


@pytest.mark.parametrize("make", [
    lambda: L.make_embed_desc(6, 9, 64, torch.zeros(6, dtype=I64)), lambda: L.make_embed_desc(6, 9, 64, torch.zeros(5, dtype=I32)),
    lambda: L.make_norm_desc(6, 64, torch.ones(64)), lambda: L.make_norm_desc(6, 64, bias=torch.ones(63, dtype=BF16)),
    lambda: L.make_norm_desc(6, 64, torch.ones(64, dtype=BF16), dtype=L.OLIVE_F32),
    lambda: L.make_sample_desc(6, 64, torch.zeros(6, dtype=BF16)), lambda: L.make_sample_desc(6, 64, torch.zeros(5)),
    lambda: L.make_sample_desc(6, 64, torch.zeros(6), temperature=torch.zeros(6, dtype=torch.float64)),
    lambda: L.make_sample_desc(6, 64, torch.zeros(6), top_k=torch.zeros(6)),
    lambda: L.make_sample_desc(6, 64, torch.zeros(6), top_p=torch.zeros(12)[::2]),
    lambda: L.make_sample_desc(6, 64, torch.zeros(6), min_p=torch.zeros(1))])
def test_descriptors_of_other_arrays(make):
    with pytest.raises(ValueError):
        make()


def test_norm_outputs_where_other_rows_lie():
    """An output may be an input itself; at its address with other strides it would overwrite rows
    that are still to be read."""
    d, one = norm_desc(), norm_desc(rows=1)
    Q = 2 * P
    for inputs in (dict(x=P, xs=0), dict(x=P, xs=128), dict(x=Q, res=P, rs=0), dict(x=Q, res=P, rs=65)):
        assert norm(d, out=P, os_=64, **inputs) == E.OLIVE_E_SHAPE
        assert norm(d, out=3 * P, os_=64, total=P, ts=64, **inputs) == E.OLIVE_E_SHAPE
    assert norm(d, x=Q, out=P, total=P, ts=64) == E.OLIVE_E_SHAPE and norm(one, x=Q, out=P, total=P) == E.OLIVE_E_SHAPE
    assert norm_backward(d, g=P, gs=0, gh=P) == E.OLIVE_E_SHAPE and norm_backward(d, g=P, gs=128, gh=P) == E.OLIVE_E_SHAPE
    assert norm_backward(d, g=Q, s=P, ss=0, gh=P) == E.OLIVE_E_SHAPE
    # (refused for what comes after: the strides are one row's, or the input's own)
    assert norm_backward(one, g=P, gs=0, gh=P, ghs=64, gw=P + 2) == E.OLIVE_E_UNSUPPORTED
    assert norm_backward(d, g=P, s=P, ss=64, gh=P, gw=P + 2) == E.OLIVE_E_UNSUPPORTED
    assert norm(d, x=Q, res=P + 1, rs=64, out=Q) == E.OLIVE_E_UNSUPPORTED
