"""olive_sample against its definition in fp64: tokens and counts exactly, log-probs to their
rounding.

The oracle tells how near a row's decisions are to falling the other way, as a share of the
masses. Both sides form the masses in 64 bits with errors of a few 2^-52 times the number of
terms, so rows that are nearer than 2^-36 may differ (none of these inputs has one: the test
says so). A log-prob is one rounding of fp32, and the logarithm's argument carries the mass's
error: 2^-24 |logp| + 2^-40.
"""
import math

import numpy as np
import pytest
import torch

from oracle import tokens_oracle as O
from paper_2609_36246_amd import _lib as L
from tests.tokens_harness import BF16, F32, U32, f64, graph_of, kind, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


def f32(v, n):
    return None if v is None else torch.tensor(np.broadcast_to(np.asarray(v, dtype=np.float32), n).copy()).cuda()


def i32(v, n):
    return None if v is None else torch.tensor(np.broadcast_to(np.asarray(v, dtype=np.int32), n).copy()).cuda()


class Sample:
    def __init__(self, logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
        n = logits.shape[0]
        self.z, self.u = logits, f32(u, n)
        self.temperature, self.top_p, self.min_p, self.top_k = f32(temperature, n), f32(top_p, n), f32(min_p, n), i32(top_k, n)
        self.desc = L.make_sample_desc(n, logits.shape[1], self.u, self.temperature, self.top_k, self.top_p, self.min_p,
                                       kind(logits.dtype))
        self.token, self.kept = (torch.full((n,), -77, dtype=torch.int32, device="cuda") for _ in range(2))
        self.logp = torch.full((n,), -77.0, device="cuda")
        self.work = torch.full((L.olive_sample_workspace(self.desc),), 0xff, dtype=torch.uint8, device="cuda")

    def call(self, stream=None):
        L.olive_sample(self.desc, self.z, self.token, self.logp, self.kept, self.work, stream=stream)

    def run(self, stream=None):
        self.call(stream)
        torch.cuda.synchronize()
        return self.token.cpu().numpy(), f64(self.logp), self.kept.cpu().numpy()

    def check(self):
        token, logp, kept = self.run()
        z = f64(self.z)
        col = lambda t, v: np.full(len(z), v) if t is None else f64(t) if t.is_floating_point() else t.cpu().numpy()  # noqa: E731
        settings = zip(col(self.u, 0), col(self.temperature, 1.0), col(self.top_k, 0), col(self.top_p, 1.0),
                       col(self.min_p, 0.0))
        for i, (u, t, k, p, m) in enumerate(settings):
            want, wlogp, n, margin = O.sample(z[i], u, t, int(k), p, m)
            assert margin > 2.0 ** -36, "row %d lies on a border: choose another input" % i
            assert (token[i], kept[i]) == (want, n), (i, u, t, k, p, m, token[i], want, kept[i], n)
            if want < 0:
                assert math.isnan(logp[i])
            else:
                assert abs(logp[i] - wlogp) <= U32 * abs(wlogp) + 2.0 ** -40 * (1 + abs(wlogp)), (i, logp[i], wlogp)
        return token


def normal(n, vocab, dtype, spread=3.0, how="plain", seed=0):
    return matrix(n, vocab, dtype, how, torch.Generator().manual_seed(seed + vocab), spread)


def uniform(n, seed=0):
    return np.random.RandomState(seed).uniform(size=n).astype(np.float32)


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(top_k=1), dict(top_k=50), dict(top_p=0.9),
            dict(min_p=0.05), dict(top_k=40, top_p=0.8), dict(temperature=1.5, top_k=300, top_p=0.95, min_p=0.01),
            dict(top_k=1 << 30, top_p=0.999), dict(top_p=0.0), dict(min_p=1.0), dict(min_p=7.0), dict(temperature=20.0, top_p=0.5),
            dict(temperature=0.01), dict(top_k=-3, top_p=2.0, min_p=-1.0), dict(temperature=1e-30, top_p=0.45),
            dict(temperature=1e30, top_k=7)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab,how", [(1, "plain"), (2, "plain"), (63, "odd"), (1000, "part"), (1025, "plain"), (4099, "odd"),
                                       (32000, "plain")])
@pytest.mark.parametrize("settings", SETTINGS, ids=lambda s: "-".join("%s_%g" % i for i in s.items()) or "plain")
def test_settings(vocab, how, dtype, settings):
    Sample(normal(5, vocab, dtype, how=how), uniform(5, vocab), **settings).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,spread", [(1, 151936, 1.0), (3, 151936, 4.0), (2, 151936, 0.01), (2, 64007, 30.0),
                                               (40, 8192, 2.0), (300, 513, 1.0), (2, 300001, 2.0), (1, 1200001, 1.0)])
def test_sizes(rows, vocab, spread, dtype):
    z = normal(rows, vocab, dtype, spread)
    for k, s in enumerate((dict(), dict(top_p=0.95), dict(top_k=1000, top_p=0.9, temperature=0.8), dict(min_p=0.02, temperature=1.3))):
        Sample(z, uniform(rows, k), **s).check()


def test_a_setting_for_each_row():
    r = np.random.RandomState(3)
    n = 64
    for dtype in (BF16, F32):
        Sample(normal(n, 5000, dtype, 4.0, seed=4), uniform(n, 5), r.choice([0.0, 0.5, 1.0, 2.0], n),
               r.choice([0, 1, 5, 60, 4999, 5000, 6000], n), r.choice([1.0, 0.3, 0.9, 0.99], n),
               r.choice([0.0, 0.0, 0.1, 0.001], n)).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [8, 1000, 40000])
def test_equal_logits(vocab, dtype):
    """Ties at every border: the lower index comes first, and equal masses add up exactly."""
    z = torch.full((6, vocab), -2.5, dtype=dtype, device="cuda")
    u = np.array([0.0, 0.1, 0.5, 0.77, 0.999, 1.0], dtype=np.float32)
    for s in (dict(), dict(top_k=3), dict(top_p=0.51), dict(min_p=1.0), dict(top_k=7, top_p=0.55)):
        got = Sample(z, u, **s)
        token, logp, kept = got.run()
        n = s.get("top_k", vocab)
        if "top_p" in s:
            c = np.arange(1, n + 1, dtype=np.float64)
            n = 1 + int((c < float(np.float32(s["top_p"])) * n).sum())
        want = np.minimum(np.floor(u.astype(np.float64) * n), n - 1)
        assert np.array_equal(kept, np.full(6, n)) and np.array_equal(token, want)
        assert np.all(np.abs(logp + math.log(n)) <= U32 * math.log(n) + 1e-12)
    z[:, vocab // 2] = 3.0                    # one above, ties below it
    for s in (dict(top_k=2), dict(top_k=5, temperature=3.0)):
        Sample(z, np.array([0.0, 0.11, 0.52, 0.771, 0.9991, 1.0], dtype=np.float32), **s).check()


def test_zeros_of_both_signs_are_equal():
    z = torch.tensor([[0.0, -0.0, 0.0, -0.0, -5.0]] * 2).cuda()
    z = torch.cat([z, -z.clone()[:, :4].flip(1), z[:, 4:]], 1)
    got = Sample(z, [0.0, 1.0], top_k=3)
    token, _, kept = got.run()
    assert kept.tolist() == [3, 3] and token.tolist() == [0, 2]
    Sample(z[:, :6].contiguous(), [0.3, 0.9], temperature=0.0).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_tokens(dtype):
    """-inf in most places, in all but one, in all; the type's lowest value instead."""
    z = normal(7, 3000, dtype, 3.0)
    z[0, ::2] = -math.inf
    z[1, 1:] = -math.inf
    z[2] = -math.inf
    z[2, 2999] = -4.0
    z[3] = -math.inf
    low = torch.finfo(dtype).min
    z[4, :2990] = low
    z[5] = low
    z[6, 100:] = -math.inf
    u = np.array([0.2, 0.99, 0.5, 0.5, 0.7, 0.0, 0.31], dtype=np.float32)
    for s in (dict(), dict(top_k=20), dict(top_k=2000), dict(top_p=0.9), dict(min_p=0.2), dict(temperature=0.0), dict(temperature=0.3)):
        token = Sample(z, u, **s).check()
        assert token[3] == -1 and token[1] == 0 and token[2] == 2999
    # what lies far below the top is kept where the cut leaves it, and drawn by u = 0 and 1 alone
    Sample(z, [0.0] * 7).check()
    Sample(z, [1.0] * 7).check()
    Sample(z, [0.0] * 7, top_k=1500).check()
    Sample(z, [1.0] * 7, top_k=1500).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_are_not_answered(dtype):
    nan, inf = math.nan, math.inf
    z = normal(9, 700, dtype)
    z[1, 5] = nan
    z[2, 699] = inf
    z[3] = -inf
    clean = Sample(z, 0.4).run()
    assert [int(t) < 0 for t in clean[0]] == [False, True, True, True] + [False] * 5
    assert np.isnan(clean[1][1:4]).all() and not clean[2][1:4].any()
    for s in (dict(u=[0.4, nan, -0.1, 1.5, inf, 0.5, 0.5, 0.5, 0.5]),
              dict(temperature=[1.0, nan, -1.0, inf, -inf, 1.0, 1.0, 1.0, 1.0]),
              dict(top_p=[0.9, nan, nan, nan, nan, 1.0, 1.0, 1.0, 1.0]), dict(min_p=[0.1, nan, nan, nan, nan, 0.0, 0.0, 0.0, 0.0])):
        u = s.pop("u", 0.4)
        got = Sample(normal(9, 700, dtype), u, **s)
        token = got.check()
        assert (token[1:5] == -1).all() and (token[[0, 5, 6, 7, 8]] >= 0).all()


def test_extremes_of_the_type():
    z = normal(4, 900, F32, 1.0)
    z[0] *= 1e38
    z[1] *= 1e-40
    z[2, 3] = torch.finfo(F32).max
    z[2, 4] = torch.finfo(F32).min
    for s in (dict(), dict(top_k=9), dict(top_p=0.7), dict(min_p=0.5), dict(temperature=1e-38), dict(temperature=3e38)):
        Sample(z, [0.1234, 0.4567, 0.7891, 0.5003], **s).check()


@pytest.mark.parametrize("vocab", [900, 40000, 151936])
def test_values_of_every_size(vocab):
    """bf16 rows that a table with a bin for each value does not hold: more powers of two than it has
    blocks, tiny values, values beyond 2^15 and below -2^15; ordinary rows between them."""
    gen = torch.Generator().manual_seed(vocab)
    n = 8
    z = torch.randn(n, vocab, generator=gen) * 3.0
    z[1] = torch.randn(vocab, generator=gen) * 2.0 ** torch.randint(-39, 14, (vocab,), generator=gen)
    z[2, ::3] = torch.randn(len(z[2, ::3]), generator=gen) * 1e-20
    z[3] *= 20000.0
    z[4, vocab // 2:] = -1e30
    z[5, : vocab - 5] = -60000.0
    z[5, vocab - 5:] = -32768.0
    z[6] = -40000.0 + 100.0 * torch.randn(vocab, generator=gen)
    z = z.to(BF16).cuda()
    for s in (dict(), dict(top_k=30), dict(top_k=vocab - 100, top_p=0.97), dict(min_p=0.03), dict(temperature=60.0, top_p=0.8),
              dict(temperature=1e4, top_k=500), dict(temperature=0.0)):
        Sample(z, uniform(n, 3), **s).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_vocabulary_of_millions(dtype):
    z = normal(1, 4500001, dtype, 1.0)
    for s in (dict(), dict(top_k=300, top_p=0.9), dict(top_p=0.5), dict(temperature=0.0)):
        Sample(z, [0.6180], **s).check()


def test_ties_across_parts():
    """Equal values at the border in every part of long rows, and runs that end inside one."""
    z = torch.full((4, 50000), -1.0, dtype=BF16, device="cuda")
    z[1, 25000:] = -2.0
    z[2, ::7] = 1.5
    z[3, 49999] = 5.0
    for s in (dict(top_k=30000), dict(top_k=7500), dict(top_k=20001, temperature=0.5), dict(top_p=0.7301)):
        Sample(z, [0.1003, 0.9502, 0.5001, 0.7503], **s).check()


def test_draws_at_both_ends_of_long_rows():
    z = normal(6, 60000, BF16, 2.0)
    for s in (dict(), dict(top_k=77), dict(top_p=0.9), dict(min_p=0.01)):
        Sample(z, [0.0, 1.0, 0.0, 1.0, 2.0 ** -24, 1.0 - 2.0 ** -24], **s).check()


def test_many_rows():
    """More rows than compute units: the counts are added by two workgroups a compute unit, and rows that
    the bins do not hold by a launch of their own."""
    z = normal(300, 20000, BF16, 3.0)
    z[5] *= 1e-15
    z[299] *= 50000.0
    u = uniform(300, 12)
    u[7], u[8] = 0.0, 1.0
    Sample(z, u, top_p=0.92, temperature=0.9).check()
    Sample(z[:, :9000].contiguous(), u, top_k=40).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_further_apart_than_32_bits_count(dtype):
    z = normal(3, 30000, dtype, 3.0)
    apart = torch.empty(2 * 1200000000 + 30000, dtype=dtype, device="cuda").as_strided((3, 30000), (1200000000, 1))
    apart.copy_(z)
    for s in (dict(), dict(top_p=0.9), dict(top_k=20, temperature=0.7)):
        want, got = Sample(z, [0.11, 0.52, 0.93], **s).run(), Sample(apart, [0.11, 0.52, 0.93], **s).run()
        assert all(np.array_equal(a, b) for a, b in zip(want, got))


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own."""
    calls = [Sample(normal(40, 40000, BF16, 2.0, seed=i), uniform(40, i), top_p=0.9) for i in range(2)]
    want = [[t.copy() for t in c.run()] for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            c.call(s)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert all(np.array_equal(a, b) for a, b in zip(w, (c.token.cpu().numpy(), f64(c.logp), c.kept.cpu().numpy())))


def test_optional_outputs_and_no_rows():
    z = normal(5, 800, BF16)
    full = Sample(z, 0.6, top_p=0.8)
    token = full.run()[0].copy()
    L.olive_sample(full.desc, z, full.kept, workspace=full.work)
    torch.cuda.synchronize()
    assert np.array_equal(full.kept.cpu().numpy(), token)
    none = Sample(torch.empty(0, 800, dtype=BF16, device="cuda"), np.zeros(0))
    none.run()


def test_a_row_that_is_read_again():
    """One row of logits for every draw (stride 0), as several rollouts of one prefix start."""
    z = normal(1, 5000, BF16).expand(50, 5000)
    token = Sample(z, uniform(50, 9), top_p=0.9).check()
    assert len(set(token.tolist())) > 5


def test_shares_of_many_draws():
    """The first 7 tokens' shares among 4000 draws of evenly spaced numbers are their
    probabilities, to two draws."""
    z = torch.tensor([[0.0, 1.0, -1.0, 2.0, 0.5, -3.0, 1.5]]).cuda()
    n = 4000
    token, _, _ = Sample(z.expand(n, 7), (np.arange(n) + 0.5) / n, temperature=0.9).run()
    p = torch.softmax(z[0].double() / 0.9, 0).cpu().numpy()
    assert np.all(np.abs(np.bincount(token, minlength=7) - n * p) <= 2)


@pytest.mark.parametrize("rows,vocab", [(3, 151936), (200, 4000)])
def test_same_bits_on_another_stream_and_in_a_graph(rows, vocab):
    a = Sample(normal(rows, vocab, BF16, 2.0), uniform(rows, 1), 0.9, 500, 0.93, 0.001)
    first = [t.copy() for t in a.run()]
    assert all(np.array_equal(x, y) for x, y in zip(first, a.run(stream=torch.cuda.Stream())))
    b = Sample(a.z, uniform(rows, 1), 0.9, 500, 0.93, 0.001)
    g = graph_of(b.call)
    for seed in (2, 3, 4):
        b.z.copy_(normal(rows, vocab, BF16, 2.0, seed=seed))
        a.u.copy_(f32(uniform(rows, seed), rows))
        b.u.copy_(a.u)
        a.top_p.fill_(0.5 + 0.1 * seed)
        b.top_p.copy_(a.top_p)
        g.replay()
        torch.cuda.synchronize()
        got = (b.token.cpu().numpy(), f64(b.logp), b.kept.cpu().numpy())
        assert all(np.array_equal(x, y) for x, y in zip(got, a.run()))
