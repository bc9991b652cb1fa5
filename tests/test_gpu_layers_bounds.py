"""The layer operators where the device arrays are not in order, at the ends of the documented
ranges, and where values are not finite."""
import pytest
import torch

from paper_2609_36246_amd import _lib as L
from tests.layers_harness import Attn

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


def filled(a, value, grad=False):
    """Output buffers that hold `value` throughout."""
    o = a.outputs(grad)
    for t in o.values():
        t.fill_(value)
    return o


def in_order(cu, b, total):
    return 0 <= cu[b] <= cu[b + 1] <= total


# (sequences, cu_q, group_seqs) with 12 query tokens: the entries of some are out of order
BROKEN = {
    "last_entry": ([0, 0, 0], [0, 4, 7, 40], [0, 3]),
    "end_of_a_group": ([0, 0, 1], [0, 4, 40, 12], [0, 2, 3]),
    "begin_of_a_group": ([0, 1, 1], [0, -3, 7, 12], [0, 1, 3]),
    "inside": ([0, 0, 0], [0, 40, 7, 12], [0, 3]),
    "more_sequences_than_there_are": ([0, 0, 1], [0, 4, 7, 12], [0, 2, 7]),
    "outside_its_group": ([0, 0, 0], [0, 4, 9, 2], [0, 3]),
}


@pytest.mark.parametrize("fill", [0x00, 0x3f, 0xff])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", list(BROKEN))
def test_offsets_out_of_order(case, dtype, fill):
    """A sequence whose own offsets are out of order is left out. The others get what is theirs,
    or NaN, and nothing that the workspace held before."""
    groups, cu, group_seqs = BROKEN[case]
    a = Attn(hq=2, hk=1, d=64, dtype=dtype, prefix=[300, 200][:max(groups) + 1],
             seqs=list(zip(groups, (8, 9, 7), (4, 3, 5))))
    a.dev["cu_q"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    a.dev["group_seqs"] = torch.tensor(group_seqs, dtype=torch.int32, device="cuda")
    desc = a.desc()
    need = L.olive_prefix_attention_workspace(desc)
    o = a.run(desc=desc, outputs=filled(a, 7.0),
              workspace=torch.full((need,), fill, dtype=torch.uint8, device="cuda"))
    # each sequence with as many queries as its offsets say, by itself
    mine = torch.zeros(12, dtype=torch.bool)
    for b in range(3):
        if not in_order(cu, b, 12) or cu[b] == cu[b + 1]:
            continue
        n = cu[b + 1] - cu[b]
        rows = slice(cu[b], cu[b + 1])
        mine[rows] = True
        got, lse = o["out"][rows], o["lse"][rows]
        if bool(torch.isnan(got).all()) and bool(torch.isnan(lse).all()):
            continue
        g = groups[b]
        s = Attn(hq=2, hk=1, d=64, dtype=dtype, prefix=[a.prefix[g]], seqs=[(0, a.seqs[b][1], n)])
        s.t["q"] = a.t["q"][rows]
        for p, at, m in (("kp", a.pstart[g], a.prefix[g]), ("vp", a.pstart[g], a.prefix[g]),
                         ("ks", a.sstart[b], a.seqs[b][1]), ("vs", a.sstart[b], a.seqs[b][1])):
            s.t[p][5:5 + m] = a.t[p][at:at + m]
        s.check({"out": got, "lse": lse})
    for t in ("out", "lse"):
        assert bool((o[t][~mine.cuda()] == 7.0).all()), t


# what the device arrays hold; of 3 sequences, the first two of one group: whose suffix rows' and
# which prefixes' gradients are NaN, whose and which are not written (their rows are unknown)
WRONG = {
    "nothing": (dict(), {}, [], [], [], []),
    "queries_over_max_q": (dict(), dict(max_q=0.9), [0], [0], [], []),
    "suffix_too_long": (dict(suffix_len=(1, 1 << 20)), {}, [], [0], [1], []),
    "suffix_outside": (dict(suffix_start=(0, 1 << 40)), {}, [], [0], [0], []),
    "prefix_outside": (dict(prefix_start=(0, -5)), {}, [0, 1], [], [], [0]),
    "prefix_too_long": (dict(prefix_len=(1, 1 << 20)), {}, [2], [], [], [1]),
    "offset_inside_a_group": (dict(cu_q=(1, 1 << 20)), {}, [0, 1], [0], [], []),
    "offset_between_groups": (dict(cu_q=(2, -4)), {}, [1, 2], [0, 1], [], []),
}


@pytest.mark.parametrize("n", [(5, 3, 7), (220, 130, 150)])
@pytest.mark.parametrize("dtype,how", [(BF16, "plain"), (BF16, "odd"), (F32, "plain")])
@pytest.mark.parametrize("case", list(WRONG))
def test_gradients_of_what_is_out_of_range(case, dtype, how, n):
    """NaN in the gradients of the keys that it concerns, where their rows are known, in no others."""
    change, stated, nan_suffix, nan_prefix, no_suffix, no_prefix = WRONG[case]
    a = Attn(hq=4, hk=1, d=64, dtype=dtype, how=how, prefix=[40, 300], grad=True,
             seqs=[(0, n[0] + 2, n[0]), (0, n[1], n[1]), (1, n[2], n[2])])
    good = a.run(grad=True)
    for k, (i, v) in change.items():
        a.dev[k][i] = v
    desc = a.desc(**{k: int(max(n) * v) for k, v in stated.items()})
    if "max_q" in stated:
        nan_suffix = [b for b in range(3) if n[b] > desc.max_q]
        nan_prefix = sorted({a.seqs[b][0] for b in nan_suffix})
    bad = a.run(grad=True, desc=desc, outputs=filled(a, 7.0, grad=True))
    rows = [("ks", b, torch.from_numpy(a.rows[b]).cuda(), nan_suffix, no_suffix) for b in range(3)]
    rows += [("kp", g, torch.arange(a.pstart[g], a.pstart[g] + a.prefix[g], device="cuda"), nan_prefix, no_prefix)
             for g in range(2)]
    for name, i, at, nans, none in rows:
        for x in ("d" + name, "dv" + name[1]):
            got = bad[x][at]
            if i in nans:
                assert bool(torch.isnan(got).all()), (x, i)
            elif i in none:
                assert bool((got == 7.0).all()), (x, i)
            elif not (case == "offset_between_groups" and (name, i) == ("ks", 0) and bool(torch.isnan(got).all())):
                # (a sequence whose group's entries do not enclose it may get NaN)
                # the same sums, cut into other parts where max_q differs
                assert torch.allclose(got.float(), good[x][at].float(), rtol=2.0 ** -6, atol=1e-2), (x, i)
    for x, used in (("ks", rows[:3]), ("kp", rows[3:])):
        keep = torch.ones(bad["d" + x].shape[0], dtype=torch.bool, device="cuda")
        for r in used:
            keep[r[2]] = False
        for y in ("d" + x, "dv" + x[1]):
            assert bool((bad[y][keep] == 7.0).all()), y


def arrays(total, prefix=0, suffix=1):
    """`total` sequences of one group with one query and `suffix` tokens each."""
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(group_seqs=i32([0, total]), cu_q=torch.arange(total + 1, dtype=torch.int32, device="cuda"),
                prefix_start=torch.zeros(1, dtype=torch.int64, device="cuda"), prefix_len=i32([prefix]),
                suffix_len=torch.full((total,), suffix, dtype=torch.int32, device="cuda"),
                suffix_start=torch.arange(total, device="cuda"), total_q=total, max_q=1, max_prefix=prefix,
                max_suffix=suffix, prefix_rows=prefix, suffix_rows=total)


def test_tokens_past_a_row_of_the_grid():
    """A wavefront a token: more of them than a dimension of a grid has threads for."""
    T = (1 << 26) + 5
    x = torch.randn(T, 1, 1, device="cuda").to(BF16)
    w = torch.full((1,), 1.5, dtype=BF16, device="cuda")
    y = torch.full_like(x, float("nan"))
    L.olive_qk_norm_rope(L.make_qk_desc(T, 1, 0, 1, weight_q=w, eps=0.25), x, None, y, None)
    f = x.float()
    want = f * torch.rsqrt(f * f + 0.25) * 1.5
    assert bool(((y.float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-30).all())


def test_rows_past_a_row_of_the_grid():
    """So many sequences and heads that the pass, and the join of its parts, take more
    workgroups than that: single tokens with one key of their own and 3 that all share."""
    B, H, D = (1 << 20) - 1, 65, 8
    rnd = lambda n: torch.randn(n, H, D, device="cuda").to(BF16)  # noqa: E731
    q, ks, vs, kp, vp = rnd(B), rnd(B), rnd(B), rnd(3), rnd(3)
    out, lse = torch.full_like(q, float("nan")), torch.full((B, H), float("nan"), device="cuda")
    desc = L.make_attn_desc(H, H, D, scale=0.5, **arrays(B, prefix=3))
    work = torch.empty(L.olive_prefix_attention_workspace(desc), dtype=torch.uint8, device="cuda")
    L.olive_prefix_attention(desc, q, kp, vp, ks, vs, out, lse, workspace=work)
    torch.cuda.synchronize()
    del work
    for at in (slice(0, 1000), slice(B // 2, B // 2 + 1000), slice(B - 1000, B)):
        k, v = (torch.cat([p[None].expand(1000, 3, H, D), s[at][:, None]], 1).double()
                for p, s in ((kp, ks), (vp, vs)))
        z = 0.5 * (q[at].double()[:, None] * k).sum(-1)
        want = (torch.softmax(z, 1)[..., None] * v).sum(1)
        # weights and outputs are rounded to bf16
        assert bool(((out[at].double() - want).abs() <= 2.0 ** -7 * v.abs().amax(1)).all())
        assert bool(((lse[at].double() - torch.logsumexp(z, 1)).abs() <= 1e-5).all())
    for part in range(0, B, 1 << 17):
        assert bool(torch.isfinite(out[part:part + (1 << 17)]).all())


@pytest.mark.parametrize("dtype,most", [(BF16, 1 << 29), (F32, 1 << 26)])
def test_keys_past_a_row_of_the_grid(dtype, most):
    """The key tiles of the longest suffixes that the sizes allow, of which few are there."""
    a = Attn(hq=4, hk=2, d=64, dtype=dtype, prefix=[30], grad=True,
             seqs=[(0, 40, 40), (0, 5, 3), (0, 1, 1), (0, 300, 200), (0, 9, 9)])
    a.check(a.run(grad=True, desc=a.desc(max_suffix=most)), grad=True)


def test_backward_rows_past_a_row_of_the_grid():
    """fp32 rows, one wavefront each in the pass before the gradients: every query sees one key,
    so dq and dk are 0 and dv is the sum of the heads' output gradients."""
    B, H = (1 << 16) + 1, 1 << 10
    rnd = lambda h: torch.randn(B, h, 1, device="cuda")  # noqa: E731
    q, do, k, v = rnd(H), rnd(H), rnd(1), rnd(1)
    desc = L.make_attn_desc(H, 1, 1, dtype=L.OLIVE_F32, scale=1.0, **arrays(B))
    out, dq = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    dk, dv = torch.full_like(k, 7.0), torch.full_like(k, 7.0)
    lse = torch.full((B, H), 7.0, device="cuda")
    work = torch.full((L.olive_prefix_attention_workspace(desc, backward=True),), 0x3f, dtype=torch.uint8,
                      device="cuda")
    L.olive_prefix_attention(desc, q, None, None, k, v, out, lse, workspace=work)
    L.olive_prefix_attention_backward(desc, q, None, None, k, v, out, lse, do, dq, None, None, dk, dv,
                                      workspace=work)
    assert bool((out == v).all()) and bool((lse - (q * k)[..., 0]).abs().amax() <= 1e-5)
    # (lse is rounded, so p is off by one unit of it at most; |do v| stays below 40)
    assert bool((dq.abs() <= 1e-4 * k.abs() + 1e-30).all())
    assert bool((dk.abs() <= 1e-4 * q.abs().sum(1, keepdim=True)).all())
    assert bool(((dv - do.sum(1, keepdim=True)).abs() <= 1e-5 * do.abs().sum(1, keepdim=True)).all())


def test_the_most_tokens_backward():
    """2^31 - 1 tokens of one element: dx = r (g w - x^2 r^2 g w)."""
    T = (1 << 31) - 1
    x, g, dx = (torch.empty(T, 1, 1, dtype=BF16, device="cuda") for _ in range(3))
    x.normal_()
    g.normal_()
    w = torch.full((1,), 1.5, dtype=BF16, device="cuda")
    desc = L.make_qk_desc(T, 1, 0, 1, weight_q=w, eps=0.25)
    L.olive_qk_norm_rope_backward(desc, x, None, g, None, dx, None)
    for at in list(range(0, T, 1 << 28)) + [T - (1 << 20)]:
        s = slice(at, min(T, at + (1 << 20)))
        y, f = x[s].double(), g[s].double() * 1.5
        r = (y * y + 0.25).rsqrt()
        # a difference of two terms of up to r |g w| in 32 bits, rounded to bf16
        want, size = r * (f - y * y * r * r * f), r * f.abs()
        assert bool(((dx[s].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size).all()), at


def test_the_longest_prefix():
    """2^31 - 1 keys: the last one, in a tile with one key less, counts once."""
    n, d = (1 << 31) - 1, 8
    k, v = (torch.zeros(n, 1, d, dtype=BF16, device="cuda") for _ in range(2))
    k[n - 1], v[n - 1] = 8.0, 1.0
    q = torch.ones(1, 1, d, dtype=BF16, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    desc = L.make_attn_desc(1, 1, d, i32([0, 1]), i32([0, 1]), torch.zeros(1, dtype=torch.int64, device="cuda"),
                            i32([n]), i32([0]), total_q=1, max_q=1, max_prefix=n, max_suffix=0, prefix_rows=n,
                            suffix_rows=0, scale=1.0)
    work = torch.empty(L.olive_prefix_attention_workspace(desc), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((1, 1), 7.0, device="cuda")
    L.olive_prefix_attention(desc, q, k, v, None, None, out, lse, workspace=work)
    # e^64 beside 2^31 times e^0
    assert abs(float(lse) - 64.0) <= 1e-4 and bool((out == 1.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("max_norm", [1.0, 1e38])
def test_norm_past_the_largest_fp32(dtype, in_place, max_norm):
    """Finite gradients whose norm is none in fp32: it is reported as infinite, and nothing is scaled."""
    g = [torch.full((n,), 3e38, device="cuda").to(dtype) for n in (5, 4000)]
    before = [x.clone() for x in g]
    outs = g if in_place else [torch.full_like(x, 7.0) for x in g]
    norm = torch.zeros(1, device="cuda")
    ctx = L.olive_grad_clip_init(g, outs)
    L.olive_grad_clip(ctx, max_norm, norm)
    torch.cuda.synchronize()
    L.olive_grad_clip_free(ctx)
    assert float(norm) == float("inf")
    assert all(torch.equal(x, y) for x, y in zip(outs, before))


def test_the_current_stream():
    """Where no stream is given it is torch's current one, on which the call runs."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert L._stream(None) == side.cuda_stream == torch.cuda.current_stream().cuda_stream
    assert L._stream(None) == torch.cuda.current_stream().cuda_stream != side.cuda_stream


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("dtype,how,d", [(BF16, "plain", 64), (BF16, "plain", 256), (BF16, "odd", 64),
                                         (BF16, "plain", 100), (F32, "plain", 64), (F32, "odd", 40),
                                         (F32, "plain", 256)])
@pytest.mark.parametrize("prefix,seqs", [([37], [(0, 70, 70), (0, 40, 9), (0, 5, 1)]),
                                         ([0, 200], [(0, 300, 300), (1, 40, 9)])])
def test_values_that_not_every_query_sees(prefix, seqs, dtype, how, d, page):
    """NaN and infinities inside a tile of keys that some rows see, and in a prefix's last row."""
    a = Attn(hq=4, hk=2, d=d, dtype=dtype, how=how, page=page, prefix=prefix, seqs=seqs, seed=13)
    for j, h, e, x in ((45, 0, 3, float("inf")), (50, 1, slice(0, d), float("nan")), (69, 0, 5, -float("inf"))):
        a.t["vs"][int(a.rows[0][j]), h, e] = x
    a.t["vp"][a.pstart[-1] + prefix[-1] - 1, 1, 2] = -float("inf")
    a.check(a.run())
    # a key: its queries get NaN, the others what they get without it
    b, j = 1, 38
    key, first = int(a.rows[b][j]), j - (seqs[b][1] - seqs[b][2])
    rows = slice(a.cu[b], a.cu[b] + first)
    a.t["ks"][key] = 0.0
    want = a.run()
    a.t["ks"][key] = float("nan")
    got = a.run()
    assert bool(torch.isnan(got["out"][a.cu[b] + first:a.cu[b + 1]]).all())
    assert bool(torch.isnan(got["lse"][a.cu[b] + first:a.cu[b + 1]]).all())
    unit = 2.0 ** -7 if dtype == BF16 else 1e-4      # (rows formed one by one round otherwise)
    x, y = got["out"][rows].double(), want["out"][rows].double()
    both = torch.isfinite(y)
    assert torch.equal(torch.isfinite(x), both) and torch.equal(x.isnan(), y.isnan())
    assert bool(((x - y).abs()[both] <= 2 * unit * (1 + y.abs()[both])).all())
    assert torch.allclose(got["lse"][rows], want["lse"][rows], rtol=1e-4, atol=1e-4)
    for c in range(len(seqs)):
        if c != b:
            s = slice(a.cu[c], a.cu[c + 1])
            assert torch.equal(torch.nan_to_num(got["out"][s], 9.0), torch.nan_to_num(want["out"][s], 9.0))


@pytest.mark.parametrize("d", [128, 127])
def test_values_keep_their_bits(d):
    """Every bf16 pattern, signalling NaNs and subnormals among them, on its way into a cache."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).cuda().view(BF16).view(512, 1, 128)[:, :, :d]
    k = torch.ones_like(v)
    ko, vo = torch.empty_like(k), torch.zeros(512, 1, 128, dtype=BF16, device="cuda")[:, :, :d]
    L.olive_qk_norm_rope(L.make_qk_desc(512, 0, 1, d), None, k, None, ko, v=v, v_out=vo)
    assert torch.equal(vo.contiguous().view(torch.int16), v.contiguous().view(torch.int16))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64), (F32, 5)])
def test_mean_squares_below_the_normal_numbers(dtype, d):
    """Without eps, heads of 1e-20: mean squares of 1e-40 (18 bits are left of them), so each
    element comes out as 1 and the gradients as those of 1 at the scale of 1e20."""
    x = torch.full((3, 2, d), 1e-20, device="cuda").to(dtype)
    x[:, :, ::2] *= -1
    w = torch.ones(d, dtype=dtype, device="cuda")
    g = torch.randn(3, 2, d, device="cuda").to(dtype)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    desc = L.make_qk_desc(3, 2, 0, d, weight_q=w, dtype=L.OLIVE_F32 if dtype == F32 else L.OLIVE_BF16, eps=0.0)
    L.olive_qk_norm_rope(desc, x, None, y, None)
    L.olive_qk_norm_rope_backward(desc, x, None, g, None, dx, None)
    r = x.double().square().mean(-1, keepdim=True).rsqrt()
    n = x.double() * r
    unit = 2.0 ** -16 + (2.0 ** -8 if dtype == BF16 else 2.0 ** -20)
    assert bool(((y.double() - n).abs() <= unit).all())
    want = r * (g.double() - n * (g.double() * n).mean(-1, keepdim=True))
    size = r * (g.double().abs() + (g.double() * n).abs().mean(-1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= unit * size).all())
