"""olive_grad_clip against the fp64 definition: the sum is formed in 64 bits, so the norm
is off by one rounding to fp32, and an output by the factor's rounding, the product's and
its type's."""
import math

import numpy as np
import pytest
import torch

from oracle import layers_oracle as O
from paper_2609_36246_amd import _lib as L
from tests.layers_harness import U16, U32, f64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


def clip(grads, max_norm, outs=None, stream=None):
    ctx = L.olive_grad_clip_init(grads, outs)
    norm = torch.full((1,), float("nan"), device="cuda")
    try:
        torch.cuda.synchronize()
        L.olive_grad_clip(ctx, max_norm, norm, stream=stream)
        torch.cuda.synchronize()
    finally:
        L.olive_grad_clip_free(ctx)
    return float(norm)


def make(sizes, seed=0, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=gen) * std).to(t).cuda() for n, t in sizes]


def check(grads, outs, norm, max_norm):
    want, n = O.clip([f64(g) for g in grads], max_norm)
    assert abs(norm - n) <= 2 * U32 * n
    for w, o in zip(want, outs):
        unit = (U16 if o.dtype == BF16 else U32) + 4 * U32
        # gradual underflow: half a step of the smallest value
        assert np.all(np.abs(f64(o) - w) <= unit * np.abs(w) + 2.0 ** -133), o.dtype


SIZES = {"one": [(1, F32)], "empty": [(0, F32), (0, BF16), (5, BF16)],
         "odd": [(1, BF16), (7, F32), (1023, BF16), (16385, F32), (40001, BF16), (3, F32)],
         "many": [(1 + 37 * i % 501, BF16 if i % 3 else F32) for i in range(700)],
         "large": [(5000003, F32), (7000001, BF16)]}


@pytest.mark.parametrize("clips", [True, False])
@pytest.mark.parametrize("sizes", list(SIZES))
def test_lists(sizes, clips):
    g = make(SIZES[sizes])
    norm64 = math.sqrt(sum(float((f64(x) ** 2).sum()) for x in g))
    most = norm64 * (0.37 if clips else 3.0)
    outs = [torch.full_like(x, float("nan")) for x in g]
    check(g, outs, clip(g, most, outs), most)
    if not clips:
        assert all(torch.equal(x, o) for x, o in zip(g, outs))
    other = [torch.full(x.shape, float("nan"), dtype=F32 if x.dtype == BF16 else BF16, device="cuda")
             for x in g]
    check(g, other, clip(g, most, other), most)
    before = [x.clone() for x in g]
    check(before, g, clip(g, most), most)
    assert all(torch.equal(x, o) for x, o in zip(g, outs))       # in place: the same bits


def test_no_gradients():
    assert clip([], 1.0) == 0.0


def test_addresses_off_16_bytes():
    base = make([(30000, F32), (30000, BF16), (30000, F32)])
    g = [base[0][1:], base[1][3:], base[2][:29000]]
    outs = [torch.empty(30000, device="cuda")[2:30000 - 0][:g[0].numel()].new_empty(g[0].numel() + 1)[1:],
            torch.empty(g[1].numel() + 5, dtype=BF16, device="cuda")[5:],
            torch.empty(29003, dtype=BF16, device="cuda")[3:]]
    check(g, outs, clip(g, 10.0, outs), 10.0)


def test_counted_only():
    g = make([(1000, F32), (2000, BF16)])
    out = torch.empty_like(g[0])
    norm = clip(g, 1.0, [out, None])
    want, n = O.clip([f64(x) for x in g], 1.0)
    assert abs(norm - n) <= 2 * U32 * n and np.allclose(f64(out), want[0], rtol=8 * U32)


@pytest.mark.parametrize("std", [1e30, 1e-30])
def test_squares_beyond_fp32(std):
    g = make([(5000, F32), (5000, BF16)], std=std)
    most = 0.5 * std
    outs = [torch.empty_like(x) for x in g]
    check(g, outs, clip(g, most, outs), most)


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_not_finite(value):
    g = make([(5000, F32), (5000, BF16)])
    g[1][4999] = value
    before = [x.clone() for x in g]
    norm = clip(g, 1.0)
    assert math.isnan(norm) if math.isnan(value) else norm == float("inf")
    for x, y in zip(g, before):
        assert torch.equal(x.view(torch.int32 if x.dtype == F32 else torch.int16),
                           y.view(torch.int32 if y.dtype == F32 else torch.int16))


def test_limits_zero_and_infinite():
    g = make([(5000, F32), (77, BF16)])
    outs = [torch.empty_like(x) for x in g]
    clip(g, 0.0, outs)
    assert all(bool((o == 0).all()) for o in outs)
    norm = clip(g, float("inf"), outs)
    assert math.isfinite(norm) and all(torch.equal(x, o) for x, o in zip(g, outs))


def test_same_bits_again_on_another_stream_and_in_a_graph():
    g = make([(3000001, F32), (500009, BF16)])
    outs = [[torch.empty_like(x) for x in g] for _ in range(2)]
    n0 = clip(g, 1.0, outs[0])
    assert n0 == clip(g, 1.0, outs[1], stream=torch.cuda.Stream())
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    ctx = L.olive_grad_clip_init(g, outs[1])
    norm = torch.empty(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        L.olive_grad_clip(ctx, 1.0, norm)
    for _ in range(3):
        g[0].mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        got, n = [o.clone() for o in outs[1]], float(norm)
        assert n == clip(g, 1.0, outs[0])
        assert all(torch.equal(x, y) for x, y in zip(got, outs[0]))
    L.olive_grad_clip_free(ctx)
