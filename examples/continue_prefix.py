"""A one-layer student on continuations of shared prefixes: rollouts, then its update.

    python examples/continue_prefix.py [--steps 4] [--tokens 48] [--prefix 300] [--rollouts 4]

The student is a frozen embedding, one attention layer with normed and rotated query and key
heads, a residual, and a vocabulary projection. Two prefixes are continued by several rollouts
each, one token of all rollouts at a time (the keys and values go to pages of a cache, each
prefix is read once for its rollouts), and the update of Eq. 1 runs on the continuations: the
layer's forward over whole continuations, the scoring with its backward, the layer's backward,
and the clipping of all gradients to a global norm. The layer's dense products are torch's;
everything else goes through the library.
"""
import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
from paper_2609_36246_amd import _lib as L  # noqa: E402

V, D, HQ, HK, HD, PAGE, EPS = 2048, 256, 4, 2, 64, 16, 1e-6
BF16 = torch.bfloat16


def angles(positions, rot=HD, base=1e4):
    """cos and sin of every position, formed in 64 bits."""
    inv = base ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return a.cos().float().cuda(), a.sin().float().cuda()


def make_student(seed=0):
    g = torch.Generator().manual_seed(seed)
    w = lambda *s, std: (torch.randn(s, generator=g) * std).to(BF16).cuda()  # noqa: E731
    return dict(embed=w(V, D, std=1.0), wqkv=w(D, (HQ + 2 * HK) * HD, std=D ** -0.5),
                gq=torch.ones(HD, dtype=BF16).cuda(), gk=torch.ones(HD, dtype=BF16).cuda(),
                wo=w(HQ * HD, D, std=(HQ * HD) ** -0.5), head=w(V, D, std=D ** -0.5))


def project(p, x):
    """Query, key and value heads: views of one product's rows."""
    qkv = (x @ p["wqkv"]).view(-1, HQ + 2 * HK, HD)
    return qkv[:, :HQ], qkv[:, HQ:HQ + HK], qkv[:, HQ + HK:]


def qk_desc(p, pos, table, **kw):
    return L.make_qk_desc(pos.shape[0], HQ, HK, HD, pos, table[0], table[1], weight_q=p["gq"],
                          weight_k=p["gk"], eps=EPS, **kw)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Prefixes:
    """Prefix tokens, packed, with their keys and values (a single layer's come from the tokens
    alone)."""

    def __init__(self, p, tokens, table):
        self.tokens = tokens                              # list of 1-D tensors
        self.len = [len(t) for t in tokens]
        self.start = [sum(self.len[:i]) for i in range(len(tokens))]
        self.x = p["embed"][torch.cat(tokens)]
        self.pos = torch.cat([torch.arange(n) for n in self.len]).int().cuda()
        self.q, self.k_raw, self.v = project(p, self.x)
        self.k = torch.empty(sum(self.len), HK, HD, dtype=BF16, device="cuda")
        L.olive_qk_norm_rope(L.make_qk_desc(len(self.pos), 0, HK, HD, self.pos, table[0], table[1],
                                            weight_k=p["gk"], eps=EPS), None, self.k_raw, None, self.k)

    def describe(self, rollouts, total_q, max_q, suffix_len, max_suffix, **kw):
        G = len(self.len)
        return L.make_attn_desc(
            HQ, HK, HD, i32([g * rollouts for g in range(G + 1)]), prefix_start=torch.tensor(self.start).cuda(),
            prefix_len=i32(self.len), suffix_len=suffix_len, total_q=total_q, max_q=max_q,
            max_prefix=max(self.len), max_suffix=max_suffix, prefix_rows=sum(self.len), **kw)


def roll_out(p, pre, table, rollouts, first, tokens):
    """Greedy continuations [B, tokens] whose first token is given, and their attention outputs."""
    B = rollouts * len(pre.len)
    pages = -(-tokens // PAGE)
    kc, vc = (torch.zeros(B * pages * PAGE, HK, HD, dtype=BF16, device="cuda") for _ in range(2))
    page_table = torch.randperm(B * pages).int().view(B, pages).cuda()
    plen = i32([n for n in pre.len for _ in range(rollouts)])
    ctx = L.olive_score_init(L.make_desc(V, D, 0, w_layout=L.OLIVE_W_VD, max_positions=B, max_seqs=1), p["head"])
    cu, cut = i32([0, B]), i32([0])
    work, logp, nxt = None, torch.empty(B, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    y, outs = [first.int()], []
    for t in range(tokens):
        x = p["embed"][y[-1].long()]
        q, k, v = project(p, x)
        slots = page_table[:, t // PAGE] * PAGE + t % PAGE
        qn, out = torch.empty(B, HQ, HD, dtype=BF16, device="cuda"), torch.empty(B, HQ, HD, dtype=BF16, device="cuda")
        L.olive_qk_norm_rope(qk_desc(p, plen + t, table, slots=slots, slot_rows=len(kc)), q, k, qn, kc, v=v, v_out=vc)
        d = pre.describe(rollouts, B, 1, torch.full_like(plen, t + 1), tokens, suffix_rows=len(kc),
                         cu_q=torch.arange(B + 1, device="cuda").int(), page_table=page_table, page_size=PAGE)
        if work is None:
            work = torch.empty(L.olive_prefix_attention_workspace(d), dtype=torch.uint8, device="cuda")
        L.olive_prefix_attention(d, qn, pre.k, pre.v, kc, vc, out, workspace=work)
        h = x + out.view(B, -1) @ p["wo"]
        L.olive_token_logprobs(ctx, L.make_batch(cu, cut, y[-1], h), logp, argmax_student=nxt)
        outs.append(out)
        y.append(nxt.clone())
    L.olive_score_free(ctx)
    return torch.stack(y[:-1], 1), torch.stack(outs, 1)


def update(p, pre, table, rollouts, y, targets, max_norm):
    """Loss (summed cross-entropy over the continuations), the attention outputs, the clipped
    gradients and their norm. y, targets: [B, n] tokens."""
    B, n = y.shape
    T = B * n
    x = p["embed"][y.reshape(-1).long()]
    q, k, v = project(p, x)
    pos = torch.cat([torch.arange(m, m + n) for m in pre.len for _ in range(rollouts)]).int().cuda()
    qd = qk_desc(p, pos, table)
    qn, kn, out = (torch.empty(T, h, HD, dtype=BF16, device="cuda") for h in (HQ, HK, HQ))
    L.olive_qk_norm_rope(qd, q, k, qn, kn)
    cu = i32([b * n for b in range(B + 1)])
    ad = pre.describe(rollouts, T, n, i32([n] * B), n, suffix_rows=T, cu_q=cu,
                      suffix_start=torch.arange(B, device="cuda") * n)
    lse = torch.empty(T, HQ, device="cuda")
    work = torch.empty(max(L.olive_prefix_attention_workspace(ad, backward=True), L.olive_qk_norm_rope_workspace(qd)),
                       dtype=torch.uint8, device="cuda")
    L.olive_prefix_attention(ad, qn, pre.k, pre.v, kn, v, out, lse=lse, workspace=work)
    o2 = out.view(T, -1)
    h = x + o2 @ p["wo"]
    # the scoring: every position of a continuation is the teacher's
    ctx = L.olive_score_init(L.make_desc(V, D, 0, w_layout=L.OLIVE_W_VD, max_positions=T, max_seqs=B,
                                         flags=L.OLIVE_FLAG_BACKWARD), p["head"])
    cut, wanted = i32([0] * B), targets.reshape(-1).int().contiguous()
    batch = L.make_batch(cu, cut, wanted, h)
    ce = torch.empty(B, device="cuda")
    L.olive_score_batch(ctx, batch, L.make_outputs(ce_per_seq=ce))
    dh, dhead = torch.empty(T, D, device="cuda"), torch.empty(V, D, device="cuda")
    L.olive_score_backward(ctx, batch, L.make_grad_outputs(1.0, 0.0, dh, dhead, reuse_forward=True))
    torch.cuda.synchronize()
    L.olive_score_free(ctx)
    # the layer
    dh = dh.to(BF16)
    dout = (dh @ p["wo"].t()).view(T, HQ, HD)
    dqkv = torch.empty(T, HQ + 2 * HK, HD, dtype=BF16, device="cuda")
    dpre = torch.zeros(len(pre.x), HQ + 2 * HK, HD, dtype=BF16, device="cuda")
    parts = lambda t: (t[:, :HQ], t[:, HQ:HQ + HK], t[:, HQ + HK:])  # noqa: E731
    (dq, dk, dv), (_, dkp, dvp) = parts(dqkv), parts(dpre)
    L.olive_prefix_attention_backward(ad, qn, pre.k, pre.v, kn, v, out, lse, dout, dq, dkp, dvp, dk, dv, workspace=work)
    gq, gk, gk_pre = (torch.empty(HD, device="cuda") for _ in range(3))
    L.olive_qk_norm_rope_backward(qd, q, k, dq, dk, dq, dk, gq, gk, workspace=work)
    pd = L.make_qk_desc(len(pre.pos), 0, HK, HD, pre.pos, table[0], table[1], weight_k=p["gk"], eps=EPS)
    L.olive_qk_norm_rope_backward(pd, None, pre.k_raw, None, dkp, None, dkp, None, gk_pre, workspace=work)
    grads = dict(wqkv=x.t() @ dqkv.view(T, -1) + pre.x.t() @ dpre.view(len(pre.x), -1), gq=gq, gk=gk + gk_pre,
                 wo=o2.t() @ dh, head=dhead)
    clip = L.olive_grad_clip_init(list(grads.values()))
    norm = torch.empty(1, device="cuda")
    L.olive_grad_clip(clip, max_norm, norm)
    L.olive_grad_clip_free(clip)
    return float(ce.sum()), out.view(B, n, HQ, HD), grads, float(norm)


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--prefix", type=int, default=300)
    ap.add_argument("--rollouts", type=int, default=4)
    ap.add_argument("--lr", type=float, default=0.05)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    p, table = make_student(), angles(a.prefix + a.tokens + 1)
    lengths = [a.prefix, max(1, a.prefix // 3)]
    tokens = [torch.randint(0, V, (n,)).cuda() for n in lengths]
    B = a.rollouts * len(lengths)
    first = torch.randint(0, V, (B,)).cuda()
    pre = Prefixes(p, tokens, table)
    y, stepwise = roll_out(p, pre, table, a.rollouts, first, a.tokens)
    # the teacher's tokens at the student's states stand in for a teacher's continuation
    targets = torch.randint(0, V, y.shape).cuda()
    losses = []
    for step in range(a.steps):
        pre = Prefixes(p, tokens, table)
        loss, out, grads, norm = update(p, pre, table, a.rollouts, y, targets, max_norm=1.0)
        if step == 0:
            off = float((out.float() - stepwise.float()).abs().max())
            print("token by token and whole continuations: outputs differ by %.4f at most" % off)
        losses.append(loss / y.numel())
        print("step %d: cross-entropy %.4f a token (log V = %.4f), gradient norm %.3f"
              % (step, losses[-1], math.log(V), norm))
        for k, g in grads.items():
            p[k] = (p[k].float() - a.lr * a.tokens * g.float()).to(BF16).contiguous()
    return losses, off


if __name__ == "__main__":
    main()
