"""The operators together, as examples/continue_prefix.py uses them: the student's gradients
against autograd in 64 bits, rollouts token by token against whole continuations, and a loss
that falls.

Bounds: each product on the way rounds its operands or result to bf16 (2^-8), a handful of
them in a row and independent, so a gradient is off by well under 2^-8 times the square root
of the roundings met by one value; 0.03 of its norm leaves a factor of two. Attention outputs
of the two ways differ by roundings of the weights and outputs: 4 units of values up to 4.
"""
import pytest
import torch

from examples import continue_prefix as E
from paper_2609_36246_amd import _lib as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


def plain_loss(w, embed, tokens, table, rollouts, y, targets):
    cos, sin = (t.double() for t in table)

    def heads(x, pos):
        qkv = (x @ w["wqkv"]).view(len(x), -1, E.HD)
        q, k, v = qkv[:, :E.HQ], qkv[:, E.HQ:E.HQ + E.HK], qkv[:, E.HQ + E.HK:]

        def turn(t, g):
            t = t / (t.pow(2).mean(-1, keepdim=True) + E.EPS).sqrt() * g
            a, b = t[..., :E.HD // 2], t[..., E.HD // 2:]
            c, s = cos[pos][:, None], sin[pos][:, None]
            return torch.cat([a * c - b * s, b * c + a * s], -1)

        return turn(q, w["gq"]), turn(k, w["gk"]), v

    loss, n = 0.0, y.shape[1]
    for b in range(len(y)):
        pre = tokens[b // rollouts]
        xp, x = embed[pre], embed[y[b].long()]
        _, kp, vp = heads(xp, torch.arange(len(pre), device="cuda"))
        q, k, v = heads(x, len(pre) + torch.arange(n, device="cuda"))
        k, v = torch.cat([kp, k]), torch.cat([vp, v])
        hidden = torch.arange(len(pre) + n, device="cuda") > len(pre) + torch.arange(n, device="cuda")[:, None]
        out = []
        for h in range(E.HQ):
            z = q[:, h] @ k[:, h // (E.HQ // E.HK)].T * E.HD ** -0.5
            out.append(torch.softmax(z.masked_fill(hidden, float("-inf")), 1) @ v[:, h // (E.HQ // E.HK)])
        hid = x + torch.cat(out, 1) @ w["wo"]
        loss = loss + torch.nn.functional.cross_entropy(hid @ w["head"].T, targets[b].long(), reduction="sum")
    return loss


def test_gradients_of_the_layer():
    torch.manual_seed(3)
    p, table = E.make_student(1), E.angles(200)
    tokens = [torch.randint(0, E.V, (n,)).cuda() for n in (90, 37)]
    y, targets = (torch.randint(0, E.V, (4, 33)).cuda() for _ in range(2))
    pre = E.Prefixes(p, tokens, table)
    loss, _, grads, norm = E.update(p, pre, table, 2, y, targets, max_norm=float("inf"))
    w = {k: v.double().requires_grad_(k != "embed") for k, v in p.items()}
    want = plain_loss(w, w["embed"], tokens, table, 2, y, targets)
    want.backward()
    assert abs(loss - want.item()) <= 1e-3 * abs(want.item())
    total = 0.0
    for k, g in grads.items():
        ref = w[k].grad
        assert float((g.double() - ref).norm()) <= 0.03 * float(ref.norm()), k
        total += float(g.double().pow(2).sum())
    assert abs(norm - total ** 0.5) <= 1e-5 * norm


def test_rollouts_and_update():
    losses, off = E.main(["--steps", "3", "--tokens", "40", "--prefix", "130", "--rollouts", "3"])
    assert off <= 4 * 4 * 2.0 ** -8
    assert losses[-1] < losses[0]
