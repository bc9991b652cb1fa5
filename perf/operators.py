"""Performance cases of the layer operators: the ones on either side of the scoring when a
student continues shared prefixes, and when it is updated on such continuations.

  rope   olive_qk_norm_rope and olive_qk_norm_rope_backward: an RMS norm of every query and
         key head, then the position rotation, in one pass; in serving the keys and values
         go to their rows of a cache in the same pass
  attn   olive_prefix_attention and olive_prefix_attention_backward: attention of sequences
         that share a prefix by groups, each with a causal suffix of its own
  clip   olive_grad_clip: the global norm over many gradients, and the gradients scaled to it

`own` chooses between the plain form (elementary torch operations in 32 bits, rounded once
at the end) and the library's calls through paper_2609_36246_amd._lib.

The integer structure of a case (lengths, pages, tensor sizes) belongs to the case and is
drawn from its `structure` number, so that its work does not depend on the seed; every
tensor value is drawn from the seed. Fields of a case:
  rope   dir "fwd" or "bwd"; seqs sequences of `len` tokens; hq, hk, d heads; rot rotated
         elements of a head; layout "half" or "pairs"; dtype; packed: queries, keys and
         values are parts of one projection's rows; cache: the tokens are written into a
         key/value cache that has so many rows more (0: no cache); reach: positions
  attn   dir "fwd" or "train" (forward, then backward); groups of seqs_lo..seqs_hi
         sequences; prefix and suffix lengths; queries: "one" (the newest token), "all" (the
         whole suffix) or "some" (the last 1..q_hi tokens); hq, hk, d, dtype; page: tokens a
         page of the suffix cache (0: packed rows)
  clip   n tensors of lo..hi values, `head` values of one more in 32 bits (0: none), dtype
         of the others; clips: whether the norm is over the limit
"""
import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------------------- cases
def _rope(**kw):
    c = dict(op="rope", dir="fwd", seqs=1, len=1, hq=16, hk=8, d=128, rot=128, layout="half",
             dtype="bf16", packed=True, cache=0, reach=8192, structure=0)
    c.update(kw)
    return c


def _attn(**kw):
    c = dict(op="attn", dir="fwd", groups=1, seqs_lo=4, seqs_hi=4, prefix_lo=4096,
             prefix_hi=4096, suffix_lo=1, suffix_hi=1024, queries="one", q_hi=1, hq=16, hk=8,
             d=128, dtype="bf16", page=0, structure=0)
    c.update(kw)
    return c


def _clip(**kw):
    c = dict(op="clip", n=8, lo=64, hi=4096, head=0, dtype="f32", clips=True, structure=0)
    c.update(kw)
    return c


def listed():
    return [
        # One token of each of 8 rollouts, keys and values written into their cache: the
        # step of a decoding loop, where the call's latency is all of it.
        _rope(name="rope_decode", seqs=8, cache=2000),
        # An update's forward over 8 rollouts of 4096 tokens (the `long_rollout` lengths) by
        # the 4096-wide model's heads.
        _rope(name="rope_forward", seqs=8, len=4096, hq=32, reach=4096),
        # Its backward for the 2048-wide student, with the gradients of the norms' weights.
        _rope(name="rope_backward", dir="bwd", seqs=8, len=4096, reach=4096),
        # A 32-bit run of a small model with a partial rotation of neighbouring pairs.
        _rope(name="rope_debug_f32", dir="bwd", seqs=7, len=111, hq=6, hk=2, d=80, rot=40,
              layout="pairs", dtype="f32", packed=False, structure=1),
        # Four rollouts from one prefix of 4096 tokens (Table 3's geometry), one token each:
        # the smallest decoding step.
        _attn(name="decode_rollouts", page=16, structure=2),
        # A serving batch: 4 long prefixes of 16 continuations each.
        _attn(name="decode_batch", groups=4, seqs_lo=16, seqs_hi=16, prefix_lo=16000,
              prefix_hi=32768, hq=32, page=16, structure=3),
        # The turns of an agent: short ragged runs of new tokens after a shared history.
        _attn(name="extend_turns", groups=3, seqs_lo=2, seqs_hi=5, prefix_lo=700,
              prefix_hi=2500, suffix_lo=90, suffix_hi=600, queries="some", q_hi=97, hq=12,
              hk=4, d=80, page=16, structure=4),
        # Ragged prompts without a prefix: a causal pass over each.
        _attn(name="prompts", groups=6, seqs_lo=1, seqs_hi=1, prefix_lo=0, prefix_hi=0,
              suffix_lo=1200, suffix_hi=6000, queries="all", d=64, structure=5),
        # The student's update on 2 prefixes of 4096 tokens with 4 continuations of 1024.
        _attn(name="update_rollouts", dir="train", groups=2, suffix_lo=1024, queries="all",
              structure=6),
        # The same in 32 bits at a size for debugging.
        _attn(name="update_debug_f32", dir="train", seqs_lo=3, seqs_hi=3, prefix_lo=150,
              prefix_hi=150, suffix_lo=30, suffix_hi=90, queries="all", hq=4, hk=2, d=64,
              dtype="f32", structure=7),
        # The gradients of a small model.
        _clip(name="clip_small", n=14, structure=8),
        # The gradients of a 2048-wide student: its vocabulary projection in 32 bits, as the
        # scoring's backward gives it, and its layers' in bf16.
        _clip(name="clip_student", n=40, lo=2048, hi=1 << 24, head=2048 * 151936,
              dtype="bf16", structure=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(16, 8), (32, 8), (16, 8), (12, 4), (8, 8), (7, 1), (6, 2)]


def _draw(rng):
    structure = rng.randrange(1 << 16)
    op = rng.choice(["rope", "decode", "decode", "some", "all", "train", "clip"])
    hq, hk = rng.choice(_HEADS)
    f32 = rng.random() < 0.2
    if op == "rope":
        d = rng.choice([128, 128, 64, 2 * rng.randrange(16, 65)])
        return _rope(dir=rng.choice(["fwd", "bwd"]), seqs=_log(rng, 1, 64), hq=hq, hk=hk, d=d,
                     len=_log(rng, 1, 4096), rot=rng.choice([d, 2 * rng.randrange(1, d // 2 + 1)]),
                     layout=rng.choice(["half", "half", "pairs"]),
                     dtype="f32" if f32 else "bf16", packed=rng.random() < 0.6,
                     cache=rng.choice([0, 1000]), reach=_log(rng, 4096, 65536),
                     structure=structure)
    if op == "clip":
        return _clip(n=_log(rng, 1, 60), lo=_log(rng, 1, 4096), hi=_log(rng, 4096, 1 << 23),
                     head=rng.choice([0, _log(rng, 1000, 1 << 28)]),
                     dtype="f32" if f32 else "bf16", clips=rng.random() < 0.8,
                     structure=structure)
    c = _attn(hq=hq, hk=hk, d=rng.choice([128, 128, 64, 8 * rng.randrange(4, 17)]),
              page=rng.choice([0, 1, 16, 16, 64]), structure=structure)
    c["groups"] = _log(rng, 1, 8)
    c["seqs_lo"] = _log(rng, 1, 8)
    c["seqs_hi"] = c["seqs_lo"] + rng.randrange(0, 9)
    c["suffix_hi"] = _log(rng, 1, 1024)
    c["suffix_lo"] = max(1, int(c["suffix_hi"] * rng.uniform(0.1, 1.0)))
    if op == "decode":
        c["prefix_hi"] = rng.choice([0, _log(rng, 64, 32768), _log(rng, 64, 32768)])
    else:
        c["prefix_hi"] = rng.choice([0, _log(rng, 16, 4096), _log(rng, 16, 4096)])
        c["queries"] = "some" if op == "some" else "all"
        c["q_hi"] = _log(rng, 2, 128) if op == "some" else 1
        if op == "train":
            c["dir"], c["page"] = "train", 0
    c["prefix_lo"] = int(c["prefix_hi"] * rng.uniform(0.3, 1.0))
    if f32 and op != "decode":
        c.update(dtype="f32", suffix_hi=min(200, c["suffix_hi"]), groups=1,
                 suffix_lo=min(200, c["suffix_lo"]), prefix_hi=min(400, c["prefix_hi"]),
                 prefix_lo=min(400, c["prefix_lo"]))
    return c


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault((c["op"], c["dir"] if "dir" in c else ""), {"bytes": 0, "flops": 0})
        for k in m:
            m[k] = max(m[k], w[k])
    while True:
        c = _draw(rng)
        w, m = work(c), most[c["op"], c["dir"] if "dir" in c else ""]
        if all(w[k] <= m[k] for k in m) and c.get("hq", 0) * c.get("d", 0) < 8192:
            return c


# -------------------------------------------------------------------- integer structure
def _attn_structure(c):
    r = np.random.RandomState(c["structure"])
    seqs = r.randint(c["seqs_lo"], c["seqs_hi"] + 1, c["groups"])
    prefix = r.randint(c["prefix_lo"], c["prefix_hi"] + 1, c["groups"])
    B = int(seqs.sum())
    suffix = r.randint(c["suffix_lo"], c["suffix_hi"] + 1, B)
    n = {"one": np.ones(B, dtype=np.int64), "all": suffix,
         "some": np.minimum(suffix, r.randint(1, c["q_hi"] + 1, B))}[c["queries"]]
    s = dict(B=B, seqs=seqs, prefix=prefix, suffix=suffix, n=n,
             group=np.repeat(np.arange(c["groups"]), seqs),
             cu_q=np.concatenate([[0], np.cumsum(n)]),
             group_seqs=np.concatenate([[0], np.cumsum(seqs)]),
             prefix_start=np.concatenate([[0], np.cumsum(prefix)])[:-1],
             prefix_rows=max(1, int(prefix.sum())))
    if c["page"]:
        pages = -(-suffix // c["page"])
        total = int(pages.sum()) + 3
        table = np.zeros((B, int(pages.max())), dtype=np.int64)
        ids, at = r.permutation(total), 0
        for b in range(B):
            table[b, :pages[b]] = ids[at:at + pages[b]]
            at += pages[b]
        s.update(table=table, suffix_rows=total * c["page"])
    else:
        s.update(suffix_start=np.concatenate([[0], np.cumsum(suffix)])[:-1],
                 suffix_rows=int(suffix.sum()))
    return s


def _clip_sizes(c):
    r = np.random.RandomState(c["structure"])
    lo, hi = min(c["lo"], c["hi"]), max(c["lo"], c["hi"])
    sizes = [(int(round(math.exp(r.uniform(math.log(lo), math.log(hi))))), c["dtype"])
             for _ in range(c["n"])]
    return ([(c["head"], "f32")] if c["head"] else []) + sizes


def _esz(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    """Each input read once and each output written once; the products of the query and key
    pairs that the mask leaves (two in the forward, five more in the backward)."""
    c = case
    if c["op"] == "clip":
        sizes = _clip_sizes(c)
        return {"bytes": sum(2 * n * _esz(t) for n, t in sizes), "flops": 3.0 * sum(n for n, _ in sizes)}
    e = _esz(c["dtype"])
    if c["op"] == "rope":
        T, H = c["seqs"] * c["len"], c["hq"] + c["hk"]
        angles = 4 * c["rot"] * min(T, c["len"] if c["len"] > 1 else T)
        if c["dir"] == "fwd":
            rows = 2 * (H + (c["hk"] if c["cache"] else 0))
            return {"bytes": e * T * c["d"] * rows + angles, "flops": 7.0 * T * H * c["d"]}
        return {"bytes": e * T * c["d"] * 3 * H + angles, "flops": 14.0 * T * H * c["d"]}
    s = _attn_structure(c)
    n, suf, pre = s["n"], s["suffix"], s["prefix"][s["group"]]
    pairs = float((n * pre + n * suf - n * (n - 1) // 2).sum())
    q = e * int(n.sum()) * c["hq"] * c["d"]
    kv = 2 * e * (int(s["prefix"].sum()) + int(suf.sum())) * c["hk"] * c["d"]
    products = 2.0 * pairs * c["hq"] * c["d"]
    if c["dir"] == "fwd":
        return {"bytes": 2 * q + kv, "flops": 2 * products}
    lse = 4 * int(n.sum()) * c["hq"]
    return {"bytes": 4 * q + 2 * kv + lse, "flops": 7 * products}


# ------------------------------------------------------------------------------ inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    x = torch.randn(shape, generator=gen, device="cuda")
    return x.mul_(std).add_(mean).to(dtype)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def _i64(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int64)).cuda()


def _rope_inputs(c, gen):
    dt, T, hq, hk, d = _dtype(c), c["seqs"] * c["len"], c["hq"], c["hk"], c["d"]
    x = {}
    if c["packed"]:
        qkv = _normal(gen, (T, hq + 2 * hk, d), dt, 1.5)
        x["q"], x["k"], x["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        x["q"], x["k"], x["v"] = (_normal(gen, (T, h, d), dt, 1.5) for h in (hq, hk, hk))
    x["wq"], x["wk"] = (_normal(gen, (d,), dt, 0.2, 1.0) for _ in range(2))
    r = np.random.RandomState(c["structure"])
    first = r.randint(0, c["reach"] - c["len"] + 1 if c["reach"] > c["len"] else 1, c["seqs"])
    if c["reach"] == c["len"]:
        first[:] = 0
    positions = (first[:, None] + np.arange(c["len"])).reshape(-1)
    x["pos"] = _i32(positions)
    inv = 1e6 ** (-torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda") * 2 / c["rot"])
    angle = torch.arange(int(positions.max()) + 1, dtype=torch.float64, device="cuda")[:, None] * inv
    x["cos"], x["sin"] = angle.cos().float(), angle.sin().float()
    if c["dir"] == "bwd":
        x["dq"], x["dk"] = _normal(gen, (T, hq, d), dt, 1e-2), _normal(gen, (T, hk, d), dt, 1e-2)
    elif c["cache"]:
        rows = T + c["cache"]
        x["slots"] = _i32(r.permutation(rows)[:T])
        x["kc"], x["vc"] = (_normal(gen, (rows, hk, d), dt) for _ in range(2))
    return x


def _attn_inputs(c, gen):
    s, dt, d = _attn_structure(c), _dtype(c), c["d"]
    n = int(s["cu_q"][-1])
    x = dict(q=_normal(gen, (n, c["hq"], d), dt, 1.5),
             kp=_normal(gen, (s["prefix_rows"], c["hk"], d), dt),
             vp=_normal(gen, (s["prefix_rows"], c["hk"], d), dt),
             ks=_normal(gen, (s["suffix_rows"], c["hk"], d), dt),
             vs=_normal(gen, (s["suffix_rows"], c["hk"], d), dt))
    if c["dir"] == "train":
        x["do"] = _normal(gen, (n, c["hq"], d), dt, 1e-2)
    x.update(cu_q=_i32(s["cu_q"]), group_seqs=_i32(s["group_seqs"]),
             prefix_len=_i32(s["prefix"]), prefix_start=_i64(s["prefix_start"]),
             suffix_len=_i32(s["suffix"]))
    if c["page"]:
        x["table"] = _i32(s["table"])
    else:
        x["suffix_start"] = _i64(s["suffix_start"])
    return x


def _clip_inputs(c, gen):
    r = np.random.RandomState(c["structure"] + 1)
    g, total = [], 0.0
    for n, t in _clip_sizes(c):
        std = 10.0 ** r.uniform(-5, -2)
        total += n * std * std
        g.append(_normal(gen, (n,), torch.bfloat16 if t == "bf16" else torch.float32, std))
    norm = math.sqrt(total)
    return dict(g=g, max_norm=0.3 * norm if c["clips"] else 10.0 * norm)


_INPUTS = {"rope": _rope_inputs, "attn": _attn_inputs, "clip": _clip_inputs}
EPS = 1e-6


class _State:
    """Inputs, output buffers, and the descriptor, workspace or plan that a program keeps."""

    def __init__(self, c, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.c, self.x, self.plan = c, _INPUTS[c["op"]](c, gen), None
        x, o = self.x, {}
        if c["op"] == "rope":
            o["q"] = torch.empty_like(x["q"], memory_format=torch.contiguous_format)
            o["k"] = x["kc"] if "kc" in x else \
                torch.empty_like(x["k"], memory_format=torch.contiguous_format)
            if "vc" in x:
                o["v"] = x["vc"]
            if c["dir"] == "bwd":
                o["wq"], o["wk"] = (torch.empty(c["d"], device="cuda") for _ in range(2))
        elif c["op"] == "attn":
            self.s = _attn_structure(c)
            o["out"] = torch.empty_like(x["q"])
            if c["dir"] == "train":
                o["lse"] = torch.empty(x["q"].shape[:2], device="cuda")
                for k in ("q", "kp", "vp", "ks", "vs"):
                    o["d" + k] = torch.zeros_like(x[k])
        else:
            o["g"] = [torch.empty_like(t) for t in x["g"]]
            o["norm"] = torch.empty(1, device="cuda")
        self.out = o

    def __del__(self):
        if getattr(self, "plan", None) and self.c["op"] == "clip":
            from paper_2609_36246_amd import _lib as L
            L.olive_grad_clip_free(self.plan)
            self.plan = None


def prepare(case, seed):
    state = _State(case, seed)
    if own:
        _plan(state)
    return state


# -------------------------------------------------------------------- the library's calls
def _plan(state):
    """The descriptor and workspace, or the list of gradients, that a program sets up once."""
    from paper_2609_36246_amd import _lib as L
    c, x, o = state.c, state.x, state.out
    kind = L.OLIVE_BF16 if c["dtype"] == "bf16" else L.OLIVE_F32
    if c["op"] == "clip":
        state.plan = L.olive_grad_clip_init(x["g"], o["g"])
        return
    if c["op"] == "rope":
        desc = state.plan = L.make_qk_desc(
            x["q"].shape[0], c["hq"], c["hk"], c["d"], x["pos"], x["cos"], x["sin"],
            weight_q=x["wq"], weight_k=x["wk"], dtype=kind, eps=EPS,
            layout=L.OLIVE_ROPE_HALF if c["layout"] == "half" else L.OLIVE_ROPE_PAIRS,
            slots=x.get("slots"), slot_rows=o["k"].shape[0] if "slots" in x else 0)
        need = L.olive_qk_norm_rope_workspace(desc) if c["dir"] == "bwd" else 0
    else:
        s = state.s
        desc = state.plan = L.make_attn_desc(
            c["hq"], c["hk"], c["d"], x["group_seqs"], x["cu_q"], x["prefix_start"],
            x["prefix_len"], x["suffix_len"], total_q=int(s["cu_q"][-1]),
            max_q=int(s["n"].max()), max_prefix=int(s["prefix"].max()),
            max_suffix=int(s["suffix"].max()), prefix_rows=s["prefix_rows"],
            suffix_rows=s["suffix_rows"], suffix_start=x.get("suffix_start"),
            page_table=x.get("table"), page_size=c["page"], dtype=kind,
            scale=1.0 / math.sqrt(c["d"]))
        need = L.olive_prefix_attention_workspace(desc, backward=c["dir"] == "train")
    state.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")


def _run_own(state):
    from paper_2609_36246_amd import _lib as L
    c, x, o, p = state.c, state.x, state.out, state.plan
    if c["op"] == "clip":
        L.olive_grad_clip(p, x["max_norm"], o["norm"])
    elif c["op"] == "rope" and c["dir"] == "fwd":
        L.olive_qk_norm_rope(p, x["q"], x["k"], o["q"], o["k"],
                             v=x["v"] if "v" in o else None, v_out=o.get("v"))
    elif c["op"] == "rope":
        L.olive_qk_norm_rope_backward(p, x["q"], x["k"], x["dq"], x["dk"], o["q"], o["k"],
                                      o["wq"], o["wk"], workspace=state.workspace)
    else:
        L.olive_prefix_attention(p, x["q"], x["kp"], x["vp"], x["ks"], x["vs"], o["out"],
                                 lse=o.get("lse"), workspace=state.workspace)
        if c["dir"] == "train":
            L.olive_prefix_attention_backward(
                p, x["q"], x["kp"], x["vp"], x["ks"], x["vs"], o["out"], o["lse"], x["do"],
                o["dq"], o["dkp"], o["dvp"], o["dks"], o["dvs"], workspace=state.workspace)
    return o


# ------------------------------------------------------------------------ the plain forms
def _rotate(x, cos, sin, c, back=False):
    """The rotation of the first `rot` elements of each head (its transpose: `back`)."""
    rot, half = c["rot"], c["rot"] // 2
    if back:
        sin = -sin
    a, b = (x[..., :half], x[..., half:rot]) if c["layout"] == "half" else \
        (x[..., 0:rot:2], x[..., 1:rot:2])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, w], -1) if c["layout"] == "half" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(state):
    c, x, o = state.c, state.x, state.out
    pos, dt = x["pos"].long(), _dtype(c)
    cos, sin = x["cos"][pos][:, None], x["sin"][pos][:, None]

    def forward(t, w):
        t = t.float()
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w.float()
        return _rotate(t, cos, sin, c).to(dt)

    def backward(t, w, grad):
        t, g = t.float(), _rotate(grad.float(), cos, sin, c, back=True)
        r = torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS)
        t = t * r
        gw = (g * t).sum((0, 1))
        g = g * w.float()
        return (r * (g - t * (g * t).mean(-1, keepdim=True))).to(dt), gw

    if c["dir"] == "bwd":
        gq, wq = backward(x["q"], x["wq"], x["dq"])
        gk, wk = backward(x["k"], x["wk"], x["dk"])
        return {"q": gq, "k": gk, "wq": wq, "wk": wk}
    q, k = forward(x["q"], x["wq"]), forward(x["k"], x["wk"])
    if not c["cache"]:
        return {"q": q, "k": k}
    at = x["slots"].long()
    o["k"][at], o["v"][at] = k, x["v"]
    return {"q": q, "k": o["k"], "v": o["v"]}


def _plain_attn(state):
    c, x, s = state.c, state.x, state.s
    B, hk, d, dt, dev = s["B"], c["hk"], c["d"], _dtype(c), "cuda"
    g = c["hq"] // hk
    scale = 1.0 / math.sqrt(d)
    P, S, N = int(s["prefix"].max()), int(s["suffix"].max()), int(s["n"].max())
    arange = lambda n: torch.arange(n, device=dev)  # noqa: E731
    cu = x["cu_q"].long()
    n, plen, slen = cu[1:] - cu[:-1], x["prefix_len"].long(), x["suffix_len"].long()
    group = torch.searchsorted(x["group_seqs"].long(), arange(B), right=True) - 1
    # padded rows: queries [B, N], keys [B, P + S], -1 where there is none
    qi = torch.where(arange(N) < n[:, None], cu[:-1, None] + arange(N), -1)
    pi = torch.where(arange(P) < plen[group][:, None], x["prefix_start"][group][:, None] + arange(P), -1)
    if c["page"]:
        t = arange(S).expand(B, S)
        at = torch.gather(x["table"].long(), 1, (t // c["page"]).clamp(max=x["table"].shape[1] - 1)) \
            * c["page"] + t % c["page"]
    else:
        at = x["suffix_start"][:, None] + arange(S)
    si = torch.where(arange(S) < slen[:, None], at, -1)
    # what a query sees: the prefix, and its suffix up to itself
    sees = torch.cat([(pi >= 0)[:, None].expand(B, N, P),
                      (si >= 0)[:, None] & (arange(S) <= (slen - n)[:, None, None] + arange(N)[:, None])], 2)
    sees = (sees & (qi >= 0)[:, :, None])[:, None, None]

    def rows(t, i):     # [B, hk, g, N, d]
        return t[i.clamp(min=0)].float().reshape(B, N, hk, g, d).permute(0, 2, 3, 1, 4)

    def keys(p, u):     # [B, hk, P + S, d]
        return torch.cat([p[pi.clamp(min=0)], u[si.clamp(min=0)]], 1).float().transpose(1, 2)

    def flat(t):        # [B, hk, g * N, last]
        return t.reshape(B, hk, g * N, t.shape[-1])

    def packed(t):      # [T, hq, ...] of [B, hk, g, N, ...]
        seq = torch.searchsorted(cu, arange(int(s["cu_q"][-1])), right=True) - 1
        t = t.permute(0, 3, 1, 2, *range(4, t.dim()))[seq, arange(len(seq)) - cu[seq]]
        return t.reshape(len(seq), c["hq"], *t.shape[3:])

    q, k, v = rows(x["q"], qi), keys(x["kp"], x["ks"]), keys(x["vp"], x["vs"])
    z = (flat(q) @ k.transpose(2, 3).contiguous()).reshape(B, hk, g, N, P + S) * scale
    z = torch.where(sees, z, -math.inf)
    top = z.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    out = (flat(p) @ v).reshape(B, hk, g, N, d)
    if c["dir"] == "fwd":
        return {"out": packed(out).to(dt)}
    lse = (top + torch.log(total))[..., 0]
    do = rows(x["do"], qi)
    dz = flat(do) @ v.transpose(2, 3).contiguous()
    dz = p * (dz.reshape(z.shape) - (do * out).sum(-1, keepdim=True)) * scale
    # a query that stands for padding has p = 0, so it adds nothing
    dq = (flat(dz) @ k).reshape(B, hk, g, N, d)
    dk = (flat(dz).transpose(2, 3).contiguous() @ flat(q)).transpose(1, 2)
    dv = (flat(p).transpose(2, 3).contiguous() @ flat(do)).transpose(1, 2)

    def back(t, like, i, part):
        w = torch.zeros_like(like, dtype=torch.float32)
        keep = (i >= 0).float()[:, :, None, None]
        return w.index_add_(0, i.clamp(min=0).reshape(-1), (t[:, part] * keep).reshape(-1, hk, d)).to(dt)

    p_, s_ = slice(0, P), slice(P, P + S)
    return {"out": packed(out).to(dt), "lse": packed(lse), "dq": packed(dq).to(dt),
            "dkp": back(dk, x["kp"], pi, p_), "dvp": back(dv, x["vp"], pi, p_),
            "dks": back(dk, x["ks"], si, s_), "dvs": back(dv, x["vs"], si, s_)}


def _plain_clip(state):
    x = state.x
    norm = torch.stack([t.float().square().sum() for t in x["g"]]).sum().sqrt()
    factor = (x["max_norm"] / (norm + EPS)).clamp(max=1.0)
    return {"g": [(t.float() * factor).to(t.dtype) for t in x["g"]], "norm": norm.reshape(1)}


_PLAIN = {"rope": _plain_rope, "attn": _plain_attn, "clip": _plain_clip}


def run(state):
    return _run_own(state) if own else _PLAIN[state.c["op"]](state)


# ---------------------------------------------------------------------------- in 64 bits
def _exact_rope(c, x):
    pos = x["pos"].long()
    half, rot = c["rot"] // 2, c["rot"]
    cos, sin = x["cos"][pos].double(), x["sin"][pos].double()
    first = torch.arange(half, device="cuda") * (1 if c["layout"] == "half" else 2)
    second = first + (half if c["layout"] == "half" else 1)

    def turn(t, sign):
        r = t.clone()
        r[..., first] = t[..., first] * cos[:, None] - sign * t[..., second] * sin[:, None]
        r[..., second] = t[..., second] * cos[:, None] + sign * t[..., first] * sin[:, None]
        return r

    def one(t, w, grad):
        t, w = t.double(), w.double()
        s = (t.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt()
        if grad is None:
            return turn(t / s * w, 1.0), None
        y = turn(grad.double(), -1.0)
        h = y * w
        return h / s - t * (h * t).sum(-1, keepdim=True) / (c["d"] * s ** 3), (y * t / s).sum((0, 1))

    (q, gq), (k, gk) = one(x["q"], x["wq"], x.get("dq")), one(x["k"], x["wk"], x.get("dk"))
    if c["dir"] == "bwd":
        return {"q": q, "k": k, "wq": gq, "wk": gk}
    if not c["cache"]:
        return {"q": q, "k": k}
    kc, vc = x["kc"].double(), x["vc"].double()
    kc[x["slots"].long()], vc[x["slots"].long()] = k, x["v"].double()
    return {"q": q, "k": kc, "v": vc}


def _exact_attn(c, x):
    """Sequence by sequence and head by head of the keys."""
    s = _attn_structure(c)
    g, d, train = c["hq"] // c["hk"], c["d"], c["dir"] == "train"
    z64 = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    o = {"out": z64(x["q"])}
    if train:
        o["lse"] = torch.zeros(x["q"].shape[:2], dtype=torch.float64, device="cuda")
        o.update({"d" + k: z64(x[k]) for k in ("q", "kp", "vp", "ks", "vs")})
    for b in range(s["B"]):
        q0, n, P, S = int(s["cu_q"][b]), int(s["n"][b]), int(s["prefix"][s["group"][b]]), int(s["suffix"][b])
        p0 = int(s["prefix_start"][s["group"][b]])
        j = np.arange(S)
        at = s["table"][b, j // c["page"]] * c["page"] + j % c["page"] if c["page"] else s["suffix_start"][b] + j
        at = torch.from_numpy(at).cuda()
        hidden = torch.arange(P + S, device="cuda") > P + S - n + torch.arange(n, device="cuda")[:, None]
        hidden = hidden.repeat_interleave(g, 0)          # rows: query, then head of the group
        for h in range(c["hk"]):
            hs = slice(h * g, (h + 1) * g)
            q = x["q"][q0:q0 + n, hs].double().reshape(n * g, d)
            k = torch.cat([x["kp"][p0:p0 + P, h], x["ks"][at, h]]).double()
            v = torch.cat([x["vp"][p0:p0 + P, h], x["vs"][at, h]]).double()
            z = (q @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse = torch.logsumexp(z, 1)
            w = torch.exp(z - lse[:, None])
            out = w @ v
            o["out"][q0:q0 + n, hs] = out.reshape(n, g, d)
            if not train:
                continue
            o["lse"][q0:q0 + n, hs] = lse.reshape(n, g)
            do = x["do"][q0:q0 + n, hs].double().reshape(n * g, d)
            dz = w * (do @ v.T - (do * out).sum(1, keepdim=True)) / math.sqrt(d)
            o["dq"][q0:q0 + n, hs] = (dz @ k).reshape(n, g, d)
            dk, dv = dz.T @ q, w.T @ do
            o["dkp"][p0:p0 + P, h] += dk[:P]
            o["dvp"][p0:p0 + P, h] += dv[:P]
            o["dks"][at, h] = dk[P:]
            o["dvs"][at, h] = dv[P:]
    return o


def _exact_clip(c, x):
    norm = math.sqrt(sum(float(torch.dot(t.double(), t.double())) for t in x["g"]))
    f = min(1.0, x["max_norm"] / (norm + EPS))
    return {"g": [t.double() * f for t in x["g"]],
            "norm": torch.tensor([norm], dtype=torch.float64)}


def exact(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = _INPUTS[case["op"]](case, gen)
    return {"rope": _exact_rope, "attn": _exact_attn, "clip": _exact_clip}[case["op"]](case, x)
