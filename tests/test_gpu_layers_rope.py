"""olive_qk_norm_rope and its backward against the fp64 definition.

Bounds: an fp32 sum of n terms is off by n units of 2^-24 of its terms' absolute sum; a
normed element takes the mean (n + 4 units), the root and three products; outputs in bf16
one unit of 2^-8 more.
"""
import numpy as np
import pytest
import torch

from oracle import layers_oracle as O
from paper_2609_36246_amd import _lib as L
from tests.layers_harness import U16, U32, f64, kind, place

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


class Case:
    def __init__(self, T=5, hq=4, hk=2, d=128, rot=None, layout="half", dtype=BF16, how="plain",
                 wq=True, wk=True, seed=0, positions=300):
        gen = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=gen).to(dtype).cuda()  # noqa: E731
        self.T, self.hq, self.hk, self.d, self.layout, self.dtype = T, hq, hk, d, layout, dtype
        self.rot = d - d % 2 if rot is None else rot
        self.q, self.k, self.v = place(rnd(T, hq, d), how), place(rnd(T, hk, d), how), rnd(T, hk, d)
        self.gq, self.gk = place(rnd(T, hq, d), how), place(rnd(T, hk, d), how)
        self.wq, self.wk = (rnd(d) if w else None for w in (wq, wk))
        self.pos = torch.randint(0, positions, (T,), generator=gen).int().cuda()
        inv = 1e4 ** (-torch.arange(self.rot // 2, dtype=torch.float64) * 2 / max(1, self.rot))
        angle = torch.arange(positions, dtype=torch.float64)[:, None] * inv
        self.cos, self.sin = angle.cos().float().cuda(), angle.sin().float().cuda()

    def desc(self, **kw):
        a = dict(positions=self.pos, cos=self.cos, sin=self.sin, weight_q=self.wq, weight_k=self.wk,
                 dtype=kind(self.dtype), eps=EPS, rot_dim=self.rot,
                 layout=L.OLIVE_ROPE_HALF if self.layout == "half" else L.OLIVE_ROPE_PAIRS)
        a.update(kw)
        return L.make_qk_desc(self.T, self.hq, self.hk, self.d, **a)

    def args(self):
        p = self.pos.cpu().numpy()
        return f64(self.cos)[p], f64(self.sin)[p], self.rot, self.layout

    def want(self, x, w):
        return O.qk_norm_rope(f64(x), None if w is None else f64(w), *self.args(), EPS)

    def want_grads(self, x, w, g):
        return O.qk_norm_rope_backward(f64(x), None if w is None else f64(w), *self.args(), EPS, f64(g))

    def unit(self):
        return (U32 if self.dtype == F32 else U16) + (self.d + 16) * U32


def close(got, want, scale, rel):
    got = f64(got)
    assert got.shape == want.shape
    err = np.abs(got - want)
    assert np.all(err <= rel * scale + 1e-30), (float(err.max()), np.argwhere(~(err <= rel * scale))[:3])


def pair_size(y):
    """A rotated element mixes two: bound it by the head's largest."""
    return np.abs(y).max(-1, keepdims=True) * 1.5


FORMS = [dict(), dict(d=64, hq=7, hk=1), dict(d=128, rot=64), dict(d=128, rot=32, layout="pairs"),
         dict(d=128, layout="pairs"), dict(d=80, rot=40), dict(d=110), dict(d=110, rot=22, layout="pairs"),
         dict(d=256, hq=2, hk=2), dict(d=1, rot=0), dict(d=3, rot=2, layout="pairs"), dict(d=255, rot=254),
         dict(d=129, rot=0), dict(d=128, dtype=F32), dict(d=256, dtype=F32, rot=128, layout="pairs"),
         dict(d=66, dtype=F32, rot=6), dict(d=128, wq=False), dict(d=96, wq=False, wk=False),
         dict(d=128, hq=4, hk=0), dict(d=128, hq=0, hk=3), dict(T=1), dict(T=1000, hq=16, hk=8)]


@pytest.mark.parametrize("how", ["plain", "packed", "odd"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join("%s%s" % i for i in f.items()) or "default")
def test_forward(form, how):
    c = Case(how=how, **form)
    qo, ko = (place(torch.full_like(t, float("nan")), how) for t in (c.q, c.k))
    L.olive_qk_norm_rope(c.desc(), c.q, c.k, qo, ko)
    for x, w, y in ((c.q, c.wq, qo), (c.k, c.wk, ko)):
        if x.numel():
            want = c.want(x, w)
            close(y, want, pair_size(want), c.unit())


@pytest.mark.parametrize("how", ["plain", "packed", "odd"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join("%s%s" % i for i in f.items()) or "default")
def test_backward(form, how):
    c = Case(how=how, **form)
    gq, gk = (place(torch.full_like(t, float("nan")), how) for t in (c.q, c.k))
    gwq, gwk = (None if w is None else torch.full((c.d,), float("nan"), device="cuda") for w in (c.wq, c.wk))
    desc = c.desc()
    work = torch.full((L.olive_qk_norm_rope_workspace(desc),), 0xff, dtype=torch.uint8, device="cuda")
    L.olive_qk_norm_rope_backward(desc, c.q, c.k, c.gq, c.gk, gq, gk, gwq, gwk, workspace=work)
    for x, w, g, got, gw in ((c.q, c.wq, c.gq, gq, gwq), (c.k, c.wk, c.gk, gk, gwk)):
        dx, dw, dw_abs = c.want_grads(x, w, g)
        if x.numel():
            # dx is r times a difference of two terms of the size of g w and of its mean with x
            r = 1.0 / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + EPS) if w is not None else 1.0
            size = r * pair_size(f64(g)) * (1.0 if w is None else np.abs(f64(w)).max()) \
                * (1.0 if w is None else 1.0 + np.abs(f64(x) * r).max(-1, keepdims=True))
            close(got, dx, np.abs(dx) + size * (c.d + 16) * U32 / c.unit(), c.unit())
        if w is not None:
            rows = c.T * max(1, x.shape[1])
            scale = dw_abs + 1.5 * np.abs(f64(g)).max(initial=0.0) * rows * 1e-3
            close(gw, dw, scale, (rows + c.d + 16) * U32)


def test_in_place_and_values():
    c = Case(T=9)
    want_q, want_k = c.want(c.q, c.wq), c.want(c.k, c.wk)
    v = torch.empty_like(c.v)
    L.olive_qk_norm_rope(c.desc(), c.q, c.k, c.q, c.k, v=c.v, v_out=v)
    close(c.q, want_q, pair_size(want_q), c.unit())
    close(c.k, want_k, pair_size(want_k), c.unit())
    assert torch.equal(v, c.v)
    g = Case(T=9)
    want = g.want_grads(g.q, g.wq, g.gq)[0]
    L.olive_qk_norm_rope_backward(g.desc(), g.q, g.k, g.gq, g.gk, g.gq, g.gk)
    close(g.gq, want, np.abs(want) + 40 * (g.d + 16) * U32 / g.unit(), g.unit())


@pytest.mark.parametrize("d", [128, 110])
def test_cache_rows(d):
    """Keys and values go to the tokens' rows; rows out of range are not written."""
    c = Case(T=6, d=d)
    kc, vc = (torch.full((10, c.hk, d), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    slots = torch.tensor([3, -1, 9, 10, 0, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    qo = torch.empty_like(c.q)
    L.olive_qk_norm_rope(c.desc(slots=slots, slot_rows=10), c.q, c.k, qo, kc, v=c.v, v_out=vc)
    want = c.want(c.k, c.wk)
    for t, row in ((0, 3), (2, 9), (4, 0)):
        close(kc[row:row + 1], want[t:t + 1], pair_size(want[t:t + 1]), c.unit())
        assert torch.equal(vc[row], c.v[t])
    rest = [1, 2, 4, 5, 6, 7, 8]
    assert bool((kc[rest] == 7.0).all()) and bool((vc[rest] == 7.0).all())
    want = c.want(c.q, c.wq)
    close(qo, want, pair_size(want), c.unit())


def test_positions_out_of_range():
    c = Case(T=5, rot=64)
    good = torch.empty_like(c.q), torch.empty_like(c.k)
    L.olive_qk_norm_rope(c.desc(), c.q, c.k, *good)
    c.pos[1], c.pos[3] = -1, c.cos.shape[0]
    bad = torch.empty_like(c.q), torch.empty_like(c.k)
    L.olive_qk_norm_rope(c.desc(), c.q, c.k, *bad)
    for g, b in zip(good, bad):
        assert bool(torch.isnan(b[[1, 3]]).all())
        assert torch.equal(g[[0, 2, 4]], b[[0, 2, 4]])


def test_values_that_are_not_finite():
    """An infinity past the rotated part stays there and turns no other element into NaN
    (rotation without a norm); a NaN stays in its head."""
    c = Case(T=4, rot=64, wq=False)
    c.q[0, 0, 100] = float("inf")
    c.q[1, 2, 5] = float("nan")
    qo, ko = torch.empty_like(c.q), torch.empty_like(c.k)
    L.olive_qk_norm_rope(c.desc(), c.q, c.k, qo, ko)
    assert float(qo[0, 0, 100]) == float("inf") and int((~torch.isfinite(qo[0])).sum()) == 1
    bad = torch.isnan(qo[1])
    assert int(bad.sum()) == 2 and bool(bad[2, 5]) and bool(bad[2, 37])
    assert bool(torch.isfinite(ko).all())


def test_no_tokens():
    c = Case(T=0)
    gwq, gwk = (torch.full((c.d,), 3.0, device="cuda") for _ in range(2))
    L.olive_qk_norm_rope(c.desc(), c.q, c.k, c.q, c.k)
    desc = c.desc()
    work = torch.empty(L.olive_qk_norm_rope_workspace(desc), dtype=torch.uint8, device="cuda")
    L.olive_qk_norm_rope_backward(desc, c.q, c.k, c.gq, c.gk, c.gq, c.gk, gwq, gwk, workspace=work)
    assert bool((gwq == 0).all()) and bool((gwk == 0).all())


def test_same_bits_again_on_another_stream_and_in_a_graph():
    c = Case(T=700, hq=8, hk=4)
    desc = c.desc()
    work = torch.empty(L.olive_qk_norm_rope_workspace(desc), dtype=torch.uint8, device="cuda")

    def call(o, stream=None):
        L.olive_qk_norm_rope(desc, c.q, c.k, o[0], o[1], stream=stream)
        L.olive_qk_norm_rope_backward(desc, c.q, c.k, c.gq, c.gk, o[2], o[3], o[4], o[5], workspace=work,
                                      stream=stream)

    new = lambda: [torch.empty_like(t) for t in (c.q, c.k, c.q, c.k)] + \
        [torch.empty(c.d, device="cuda") for _ in range(2)]  # noqa: E731
    a, b, g = new(), new(), new()
    call(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(b, side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(g)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        call(a)
        torch.cuda.synchronize()
        for x, y, z in zip(a, b, g):
            assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_gradients_against_differences(layout):
    c = Case(T=3, hq=2, hk=1, d=16, rot=12, layout=layout, dtype=F32)
    desc = c.desc()
    o = [torch.empty_like(c.q), torch.empty_like(c.k), torch.empty(16, device="cuda"),
         torch.empty(16, device="cuda")]
    work = torch.empty(L.olive_qk_norm_rope_workspace(desc), dtype=torch.uint8, device="cuda")
    L.olive_qk_norm_rope_backward(desc, c.q, c.k, c.gq, c.gk, *o, workspace=work)
    x, w, g = f64(c.q), f64(c.wq), f64(c.gq)
    loss = lambda x, w: float((O.qk_norm_rope(x, w, *c.args(), EPS) * g).sum())  # noqa: E731
    r, h = np.random.RandomState(1), 1e-5
    for got, base, f in ((f64(o[0]), x, lambda y: loss(y, w)), (f64(o[2]), w, lambda y: loss(x, y))):
        way = r.randn(*base.shape)
        want = (f(base + h * way) - f(base - h * way)) / (2 * h)
        assert abs(float((got * way).sum()) - want) <= 1e-5 * float(np.abs(got * way).sum()) + 1e-6
