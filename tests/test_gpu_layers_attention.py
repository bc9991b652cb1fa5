"""olive_prefix_attention and its backward against the fp64 definition.

Tolerances (tests/layers_harness.py, Attn.relative) follow from the roundings that the
operator makes and were set before the first run.
"""
import numpy as np
import pytest
import torch

from oracle import layers_oracle as O
from paper_2609_36246_amd import _lib as L
from tests.layers_harness import Attn, f64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


def one(prefix, suffixes):
    """Single-token queries: (group, suffix length) pairs."""
    return dict(prefix=prefix, seqs=[(g, s, 1) for g, s in suffixes])


SHAPES = {
    "one_key": one([0], [(0, 1)]),
    "prefix_only": dict(prefix=[1], seqs=[(0, 0, 1)]),
    "decode": one([300], [(0, 1), (0, 17), (0, 64), (0, 65)]),
    "decode_long": one([5003], [(0, 700), (0, 1), (0, 129)]),
    "decode_groups": one([40, 0, 129], [(0, 5), (0, 66), (1, 31), (2, 1), (2, 2), (2, 300)]),
    "decode_alone": one([0, 0, 0], [(0, 3), (1, 2000), (2, 32)]),
    "many_in_a_group": one([190], [(0, 1 + i % 9) for i in range(40)]),
    "extend": dict(prefix=[77, 500], seqs=[(0, 40, 7), (0, 130, 33), (1, 64, 64), (1, 90, 2)]),
    "prompts": dict(prefix=[0, 0], seqs=[(0, 200, 200), (1, 131, 131)]),
    "update": dict(prefix=[260], seqs=[(0, 150, 150), (0, 33, 33), (0, 1, 1)]),
    # more queries than suffix tokens: the first ones see the prefix alone, or nothing
    "early_queries": dict(prefix=[9, 0], seqs=[(0, 3, 8), (1, 2, 6), (1, 0, 4)]),
    # sequences without queries, groups without sequences
    "absent": dict(prefix=[12, 50, 0, 33], seqs=[(0, 4, 0), (0, 20, 3), (3, 7, 7), (3, 0, 0)]),
    # more query rows than any tile, fewer keys than any tile
    "tall": dict(prefix=[3], seqs=[(0, 2, 2)] * 70),
}
HEADS = [(4, 2, 64, BF16), (2, 2, 128, BF16), (7, 1, 128, BF16), (6, 2, 80, BF16), (4, 1, 112, BF16),
         (3, 3, 40, BF16), (4, 2, 96, BF16), (4, 2, 24, BF16), (2, 1, 8, BF16), (4, 2, 256, BF16), (2, 1, 100, BF16), (2, 1, 1, BF16), (4, 2, 64, F32),
         (7, 1, 36, F32), (2, 2, 256, F32)]


@pytest.mark.parametrize("hq,hk,d,dtype", HEADS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_forward(shape, hq, hk, d, dtype):
    a = Attn(hq=hq, hk=hk, d=d, dtype=dtype, **SHAPES[shape])
    a.check(a.run())


@pytest.mark.parametrize("page", [1, 3, 16, 64])
@pytest.mark.parametrize("shape", ["one_key", "decode", "decode_long", "decode_groups", "extend",
                                   "prompts", "early_queries", "absent", "tall"])
def test_pages(shape, page):
    a = Attn(hq=8, hk=2, d=128, page=page, **SHAPES[shape])
    a.check(a.run())


@pytest.mark.parametrize("how", ["packed", "heads", "odd"])
@pytest.mark.parametrize("shape", ["decode_groups", "extend", "update"])
def test_layouts(shape, how):
    a = Attn(hq=6, hk=2, d=64, how=how, grad=True, **SHAPES[shape])
    a.check(a.run(grad=True), grad=True)


@pytest.mark.parametrize("hq,hk,d,dtype", HEADS)
@pytest.mark.parametrize("shape", ["one_key", "prefix_only", "decode_groups", "extend", "prompts",
                                   "update", "early_queries", "absent", "tall"])
def test_backward(shape, hq, hk, d, dtype):
    a = Attn(hq=hq, hk=hk, d=d, dtype=dtype, grad=True, **SHAPES[shape])
    a.check(a.run(grad=True), grad=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_queries(dtype):
    """Nothing to do forward; the gradients of every key are zero."""
    a = Attn(prefix=[40], seqs=[(0, 5, 0), (0, 0, 0)], dtype=dtype, grad=True)
    a.check(a.run(grad=True), grad=True)


@pytest.mark.parametrize("shape,n", [("update", 700), ("prompts", 1100)])
def test_longer_runs(shape, n):
    """Several tiles of rows and keys in every direction."""
    kw = dict(prefix=[900], seqs=[(0, n, n), (0, n // 3, n // 3)]) if shape == "update" else \
        dict(prefix=[0], seqs=[(0, n, n)])
    a = Attn(hq=4, hk=2, d=128, grad=True, seed=3, **kw)
    a.check(a.run(grad=True), grad=True)


@pytest.mark.parametrize("hq,hk", [(3, 3), (4, 2), (4, 1)])
def test_ragged_runs_of_many_tiles(hq, hk):
    """More tiles of rows and of keys than are taken in one go, and sequences that lack most of them."""
    a = Attn(hq=hq, hk=hk, d=64, prefix=[0, 2200, 0], seqs=[(0, 2300, 2300), (1, 129, 129), (1, 1, 1), (2, 700, 700)],
             grad=True, seed=12)
    a.check(a.run(grad=True), grad=True)


def test_peaked_rows():
    """Weights that underflow beside ones near 1, and a maximum that grows along the keys."""
    a = Attn(hq=4, hk=2, d=64, prefix=[400], seqs=[(0, 200, 200), (0, 90, 1)], std=4.0, grad=True, seed=5)
    ramp = torch.linspace(0.05, 1.0, a.t["kp"].shape[0], device="cuda")[:, None, None].to(BF16)
    a.t["kp"] *= ramp
    a.check(a.run(grad=True), grad=True)


@pytest.mark.parametrize("seqs,prefix", [([(0, 70, 70)], [0]), ([(0, 40, 40), (0, 66, 20)], [130])])
def test_values_that_a_query_does_not_see(seqs, prefix):
    """NaN and infinite keys and values of the newest token reach the queries that see it only."""
    a = Attn(hq=4, hk=2, d=128, prefix=prefix, seqs=seqs, seed=6)
    last = int(a.rows[0][-1])
    a.t["vs"][last, 0, 3] = float("inf")
    a.t["vs"][last, 1] = NAN
    a.check(a.run())
    a.t["ks"][last] = NAN
    out = a.run()["out"][a.cu[0]:a.cu[1]]
    assert bool(torch.isnan(out[-1]).all()) and bool(torch.isfinite(out[:-1]).all())


def test_scores_of_minus_infinity():
    """A query all of whose scores are -inf counts as one that sees nothing."""
    a = Attn(hq=2, hk=2, d=64, prefix=[20], seqs=[(0, 9, 9)], seed=7)
    a.t["q"][4] = 3e38
    a.t["kp"][a.pstart[0]:a.pstart[0] + 20] = -3e38
    a.t["ks"][torch.from_numpy(a.rows[0]).cuda()] = -3e38
    o = a.run()
    assert bool((o["out"][4] == 0).all()) and bool((o["lse"][4] == -float("inf")).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_out_of_range_arrays(dtype):
    """Bad device contents give NaN to the sequences they concern, and no other."""
    kw = dict(hq=4, hk=2, d=64, dtype=dtype, prefix=[30, 50], seqs=[(0, 20, 5), (0, 9, 1), (1, 7, 7)])

    def nan_rows(a, **change):
        good = a.run()
        for k, v in change.items():
            a.dev[k] = torch.tensor(v, dtype=a.dev[k].dtype, device="cuda")
        desc = a.desc()
        bad = a.run(desc=desc)
        is_nan = torch.isnan(bad["out"]).flatten(1)
        rows = [bool(is_nan[a.cu[b]:a.cu[b + 1]].all()) for b in range(3)]
        for b in range(3):
            if not rows[b]:
                s = slice(a.cu[b], a.cu[b + 1])
                assert torch.equal(bad["out"][s], good["out"][s])
                assert torch.equal(bad["lse"][s], good["lse"][s])
        return rows

    a = Attn(**kw)
    assert nan_rows(a, prefix_len=[30, 51]) == [False, False, True]      # over max_prefix = 50
    assert nan_rows(Attn(**kw), prefix_len=[30, -1]) == [False, False, True]
    assert nan_rows(Attn(**kw), prefix_start=[-1, a.pstart[1]]) == [True, True, False]
    assert nan_rows(Attn(**kw), prefix_start=[a.pstart[0], a.prefix_rows - 49]) == [False, False, True]
    assert nan_rows(Attn(**kw), suffix_len=[20, 21, 7]) == [False, True, False]
    assert nan_rows(Attn(**kw), suffix_len=[20, 9, -7]) == [False, False, True]
    assert nan_rows(Attn(**kw), suffix_start=[a.sstart[0], 1 << 40, a.sstart[2]]) == [False, True, False]
    p = Attn(page=16, **kw)
    table = p.table.copy()
    table[0, 1] = p.suffix_rows // 16
    assert nan_rows(p, page_table=table) == [True, False, False]
    p = Attn(page=16, **kw)
    table = p.table.copy()
    table[2, 0] = -1
    assert nan_rows(p, page_table=table) == [False, False, True]


@pytest.mark.parametrize("seqs,max_q", [([(0, 9, 1), (0, 30, 3), (0, 4, 1)], 1),
                                        ([(0, 400, 300), (0, 300, 200)], 250)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_queries_than_stated(seqs, max_q, dtype):
    """A sequence with more than max_q queries gets NaN in all of them, the others what is theirs."""
    a = Attn(hq=4, hk=2, d=64, dtype=dtype, prefix=[50], seqs=seqs, grad=True)
    good, bad = a.run(), a.run(grad=True, desc=a.desc(max_q=max_q))
    for b, (_, _, n) in enumerate(seqs):
        s = slice(a.cu[b], a.cu[b + 1])
        for k in ("out", "lse") + (("dq",) if n > max_q else ()):
            if n > max_q:
                assert bool(torch.isnan(bad[k][s]).all()), (b, k)
        if n <= max_q:
            ref = a.reference()[b]
            assert np.all(np.abs(f64(bad["out"][s]) - ref["out"]) <= 0.05 * ref["out_abs"] + 1e-3)
            assert torch.allclose(bad["lse"][s], good["lse"][s], rtol=1e-5)


@pytest.mark.parametrize("groups,dtype", [(64, BF16), (131, BF16), (64, F32)])
def test_many_groups(groups, dtype):
    """More groups and sequences than a wavefront looks through at once."""
    r = np.random.RandomState(1)
    seqs = [(g, int(r.randint(1, 9)), 1) for g in range(groups) for _ in range(r.randint(0, 5))]
    a = Attn(hq=2, hk=1, d=64, dtype=dtype, prefix=[int(x) for x in r.randint(0, 40, groups)], seqs=seqs)
    a.check(a.run())


def test_many_sequences():
    a = Attn(hq=1, hk=1, d=64, prefix=[3, 5], seqs=[(i // 2600, 1 + i % 3, 1) for i in range(5200)], spare=0)
    a.check(a.run())
    a = Attn(hq=1, hk=1, d=64, prefix=[0] * 4200, seqs=[(i, 1 + i % 3, 1) for i in range(4200)], spare=0)
    a.check(a.run())


def test_workspace_of_the_largest_call_serves_the_others():
    need = lambda **k: L.olive_prefix_attention_workspace(Attn(hq=8, hk=2, d=128, **k).desc(), backward=True)  # noqa: E731
    most = need(prefix=[400], seqs=[(0, 64, 64)] * 4)
    assert all(need(**SHAPES[s]) <= most for s in ("one_key", "decode", "decode_long", "decode_groups", "extend"))


def test_workspace_holds_more_queries_than_stated():
    """Nothing is written past the workspace where a sequence has more queries than max_q."""
    a = Attn(hq=4, hk=2, d=64, prefix=[20000], seqs=[(0, 5, 3000)], seed=11)
    desc = a.desc(max_q=1)
    need = L.olive_prefix_attention_workspace(desc)
    room = torch.full((need + (64 << 20),), 0xa5, dtype=torch.uint8, device="cuda")
    o = a.run(desc=desc, workspace=room[:need])
    torch.cuda.synchronize()
    assert bool((room[need:] == 0xa5).all())
    assert bool(torch.isnan(o["out"]).all()) and bool(torch.isnan(o["lse"]).all())


def test_query_offsets_out_of_order():
    """A sequence whose query rows are not in [0, total_q] is left out."""
    a = Attn(hq=2, hk=1, d=64, prefix=[30], seqs=[(0, 8, 4), (0, 9, 3), (0, 5, 5)])
    good = a.run()
    a.dev["cu_q"] = torch.tensor([0, 4, 40, 12], dtype=torch.int32, device="cuda")
    bad = a.run(desc=a.desc())
    assert torch.equal(bad["out"][:4], good["out"][:4])
    assert bool(torch.isnan(bad["out"][4:]).all())          # as the harness filled it


def test_long_cache_offsets():
    """Rows whose offsets pass 32 bits: a cache of more than 4 GiB, used at its end."""
    hk, d, page = 8, 128, 64
    pages = (5 << 30) // (page * hk * d * 2)
    a = Attn(hq=8, hk=hk, d=d, page=page, prefix=[20], seqs=[(0, 150, 3)], seed=9)
    ref = a.reference()
    big = {}
    for name in ("ks", "vs"):
        big[name] = torch.empty((pages * page, hk, d), dtype=BF16, device="cuda")
        big[name][-a.suffix_rows:] = a.t[name]
    a.dev["page_table"] = a.dev["page_table"] + (pages - a.suffix_rows // page)
    a.dev["page_table"][a.dev["page_table"] >= pages] = 0
    a.t.update(big)
    a.suffix_rows = pages * page
    a.check(a.run(), ref)
    del big
    # and a packed prefix at the end of such a buffer
    b = Attn(hq=8, hk=hk, d=d, prefix=[400], seqs=[(0, 3, 3)], seed=10, grad=True)
    ref = b.reference(grad=True)
    rows = (5 << 30) // (hk * d * 2)
    shift = rows - b.prefix_rows
    for name in ("kp", "vp"):
        t = torch.empty((rows, hk, d), dtype=BF16, device="cuda")
        t[shift:] = b.t[name]
        b.t[name] = t
    b.dev["prefix_start"] = b.dev["prefix_start"] + shift
    b.prefix_rows = rows
    o = b.run(grad=True)
    for name in ("dkp", "dvp"):
        o[name] = o[name][shift:]
    b.check(o, ref, grad=True)


def test_same_bits_on_another_stream_and_again():
    a = Attn(hq=8, hk=2, d=128, prefix=[900, 40], seqs=[(0, 200, 200), (0, 70, 70), (1, 33, 33)], grad=True)
    first = {k: v.clone() for k, v in a.run(grad=True).items()}
    side = torch.cuda.Stream()
    again = a.run(grad=True, stream=side)
    side.synchronize()
    for k in first:
        assert torch.equal(first[k], again[k]), k
    d = Attn(hq=8, hk=2, d=128, page=16, **SHAPES["decode_long"])
    first, again = d.run(), d.run()
    assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])


@pytest.mark.parametrize("grad", [False, True])
def test_graph_replays(grad):
    shape = SHAPES["update"] if grad else SHAPES["decode_long"]
    a = Attn(hq=8, hk=2, d=128, page=0 if grad else 16, grad=grad, **shape)
    desc, o = a.desc(), a.outputs(grad)
    work = torch.empty(L.olive_prefix_attention_workspace(desc, backward=grad), dtype=torch.uint8,
                       device="cuda")
    a.run(grad, desc, outputs=o, workspace=work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(grad, desc, outputs=o, workspace=work)
    for i in range(3):
        a.t["q"].copy_(torch.randn(a.t["q"].shape, device="cuda").to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in o.items()}
        eager = a.run(grad, desc)
        torch.cuda.synchronize()
        for k in got:
            assert torch.equal(got[k], eager[k]), (i, k)


def test_shorter_than_the_bounds():
    """max_q, max_prefix and max_suffix may be larger than what the arrays hold."""
    a = Attn(hq=8, hk=2, d=128, prefix=[100, 5], seqs=[(0, 30, 1), (0, 3, 1), (1, 9, 1)])
    a.check(a.run(desc=a.desc(max_q=50, max_prefix=20000, max_suffix=9000)))
    a.check(a.run(desc=a.desc(max_prefix=20000)))
    b = Attn(hq=4, hk=2, d=64, prefix=[100], seqs=[(0, 30, 30), (0, 3, 3)], grad=True)
    b.check(b.run(grad=True, desc=b.desc(max_q=600, max_prefix=3000, max_suffix=700)), grad=True)


def test_gradients_against_differences():
    """fp32 gradients against central differences of the fp64 definition."""
    a = Attn(hq=4, hk=2, d=32, dtype=F32, prefix=[11, 4], seqs=[(0, 7, 5), (0, 3, 3), (1, 4, 6)], grad=True,
             std=0.7)
    o = a.run(grad=True)
    r = np.random.RandomState(0)

    def loss():
        return sum(float((s["out"] * s["do"]).sum()) for s in a.reference(grad=True))

    for name in ("q", "kp", "vp", "ks", "vs"):
        used = np.isfinite(f64(a.t[name]))
        way = np.where(used, r.randn(*used.shape), 0.0)
        base, h = a.t[name], 1e-4
        a.t[name] = base.double() + h * torch.from_numpy(way).cuda()
        up = loss()
        a.t[name] = base.double() - h * torch.from_numpy(way).cuda()
        down = loss()
        a.t[name] = base
        got = float((np.where(used, f64(o["d" + name]), 0.0) * way).sum())
        # the difference is off by h^2 times a third derivative, the sum by fp32's rounding
        size = float(np.abs(np.where(used, f64(o["d" + name]), 0.0) * way).sum())
        assert abs(got - (up - down) / (2 * h)) <= 1e-5 * size + 1e-6, name


def test_oracle_tells_a_wrong_mask():
    """The bounds see a mask that is one key off (planted in the oracle's inputs)."""
    a = Attn(hq=2, hk=1, d=64, prefix=[20], seqs=[(0, 30, 4)])
    o = a.run()
    ref = a.reference()
    for s in ref:
        s["k"], s["v"] = s["k"][:-1], s["v"][:-1]
    with pytest.raises(AssertionError):
        a.check(o, O.attention(ref, a.scale, a.hq, a.hk))
