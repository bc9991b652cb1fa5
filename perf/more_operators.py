"""Performance cases of the token operators: the way from tokens to rows, between the layers,
and from logits back to tokens, for rollouts (forward) and for the update on them (backward).

  embed   olive_embed and olive_embed_backward: rows of an embedding table, scaled; the
          table's gradient by sorted tokens, written whole or added to one that is there
          (the vocabulary projection's, where the two share their weight)
  norm    olive_row_norm and olive_row_norm_backward: the residual added, then a layer norm
          or an RMS norm of each row; the gradients of the rows and of weight and bias
  sample  olive_sample: the next token of every row of logits with temperature, top-k, top-p
          and min-p from given uniform numbers, its log-prob, and how many tokens were kept

`own` chooses between the plain form (elementary torch operations in 32 bits, in 64 for the
distribution that a token is drawn from) and the library's calls through
paper_2609_36246_amd._lib.

The integer structure of a case (tokens, per-row sampling settings) belongs to the case and is
drawn from its `structure` number, so that its work does not depend on the seed; every
tensor value is drawn from the seed. Fields of a case:
  embed   dir "fwd" or "bwd"; tokens, vocab, d; dtype of the rows; ids "text" (a few tokens
          are most of them) or "uniform"; pad: share of padded tokens (-1); scaled: by the
          root of d; grad: dtype of the table's gradient; add: it is added to what is there
  norm    dir; rows, d, dtype; kind "rms" or "layer"; bias; residual
  sample  rows, vocab, dtype; spread: the logits' standard deviation; masked: share of
          logits at -inf; temp, top_k, top_p, min_p: one setting of all rows (1, 0, 1 and 0:
          not passed), or mixed: settings of their own, greedy rows among them
"""
import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------------------- cases
def _embed(**kw):
    c = dict(op="embed", dir="fwd", tokens=8, vocab=151936, d=2048, dtype="bf16", ids="text", pad=0.0,
             scaled=False, grad="f32", add=False, structure=0)
    c.update(kw)
    return c


def _norm(**kw):
    c = dict(op="norm", dir="fwd", rows=8, d=2048, dtype="bf16", kind="rms", bias=False, residual=True, structure=0)
    c.update(kw)
    return c


def _sample(**kw):
    c = dict(op="sample", dir="fwd", rows=4, vocab=151936, dtype="bf16", spread=4.0, masked=0.0, temp=1.0, top_k=0,
             top_p=1.0, min_p=0.0, mixed=False, structure=0)
    c.update(kw)
    return c


def listed():
    return [
        # The newest tokens of 8 rollouts: the start of a decoding step.
        _embed(name="embed_decode"),
        # An update's input rows: 8 rollouts of 4096 tokens (the `long_rollout` lengths), some
        # of them padding.
        _embed(name="embed_forward", tokens=32768, pad=0.1, structure=1),
        # Their gradient, added to the vocabulary projection's (a student with tied weights).
        _embed(name="embed_grad_tied", dir="bwd", tokens=32768, pad=0.1, add=True, structure=1),
        # The whole gradient of an embedding of its own (the `large_vocab` student's width).
        _embed(name="embed_grad_table", dir="bwd", tokens=8192, d=1536, scaled=True, structure=2),
        # A decoding step's norm between two layers.
        _norm(name="norm_decode"),
        # The norm over an update's rows at the 4096-wide model.
        _norm(name="norm_forward", rows=32768, d=4096),
        # Its backward at the student's width, with the weight's gradient and the residual's.
        _norm(name="norm_backward", dir="bwd", rows=32768),
        # A small model with layer norms in 32 bits, as one debugs a bf16 run against.
        _norm(name="norm_debug_f32", dir="bwd", rows=777, d=1600, dtype="f32", kind="layer", bias=True,
              residual=False),
        # The next token of 4 rollouts at temperature 1 (Table 3), nothing cut off.
        _sample(name="sample_rollouts", structure=3),
        # A serving batch whose requests bring their own settings, with forbidden tokens.
        _sample(name="sample_batch", rows=64, mixed=True, masked=0.05, structure=4),
        # 32-bit logits of a small vocabulary with the usual cuts.
        _sample(name="sample_debug_f32", rows=8, vocab=32000, dtype="f32", spread=3.0, temp=0.7, top_k=50, top_p=0.95,
                structure=5),
        # One step of 512 rollouts with a nucleus.
        _sample(name="sample_many", rows=512, top_p=0.95, structure=6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    structure = rng.randrange(1 << 16)
    op = rng.choice(["embed", "grad", "grad", "norm", "norm", "sample", "sample", "sample"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    d = rng.choice([1024, 2048, 4096, 64 * rng.randrange(2, 64), _log(rng, 60, 5200)])
    vocab = rng.choice([151936, 32000, _log(rng, 1000, 152000)])
    if op in ("embed", "grad"):
        return _embed(dir="fwd" if op == "embed" else "bwd", tokens=_log(rng, 1, 32768), vocab=vocab, d=d, dtype=dtype,
                      ids=rng.choice(["text", "text", "uniform"]), pad=rng.choice([0.0, 0.2]),
                      scaled=rng.random() < 0.3, grad=rng.choice(["f32", "f32", "bf16"]), add=rng.random() < 0.5,
                      structure=structure)
    if op == "norm":
        kind = rng.choice(["rms", "rms", "layer"])
        return _norm(dir=rng.choice(["fwd", "bwd"]), rows=_log(rng, 1, 32768), d=d, dtype=dtype, kind=kind,
                     bias=kind == "layer" and rng.random() < 0.7, residual=rng.random() < 0.6, structure=structure)
    return _sample(rows=_log(rng, 1, 512), vocab=vocab, dtype=dtype, spread=rng.choice([1.0, 2.0, 4.0, 8.0]),
                   masked=rng.choice([0.0, 0.0, 0.05, 0.9]), temp=rng.choice([1.0, 1.0, 0.6, 1.3]),
                   top_k=rng.choice([0, 0, _log(rng, 1, 1000)]),
                   top_p=rng.choice([1.0, round(rng.uniform(0.5, 0.99), 3)]),
                   min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.3), 3)]), mixed=rng.random() < 0.3,
                   structure=structure)


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault((c["op"], c["dir"]), {"bytes": 0, "flops": 0})
        for k in m:
            m[k] = max(m[k], w[k])
    while True:
        c = _draw(rng)
        w, m = work(c), most[c["op"], c["dir"]]
        if all(w[k] <= m[k] for k in m):
            return c


# -------------------------------------------------------------------- integer structure
def _tokens(c):
    r = np.random.RandomState(c["structure"])
    if c["ids"] == "text":       # the n-th most frequent token is one of n, frequent ones first
        ids = np.exp(r.uniform(0, math.log(c["vocab"] + 1), c["tokens"])).astype(np.int64) - 1
    else:
        ids = r.randint(0, c["vocab"], c["tokens"])
    ids = np.clip(ids, 0, c["vocab"] - 1)
    ids[r.uniform(size=c["tokens"]) < c["pad"]] = -1
    return ids


def _settings(c):
    """Per-row temperature, top_k, top_p and min_p (None: not passed)."""
    n = c["rows"]
    if not c["mixed"]:
        return (None if c["temp"] == 1.0 else np.full(n, c["temp"]), np.full(n, c["top_k"]) if c["top_k"] else None,
                None if c["top_p"] == 1.0 else np.full(n, c["top_p"]), np.full(n, c["min_p"]) if c["min_p"] else None)
    r = np.random.RandomState(c["structure"])
    temp = np.where(r.uniform(size=n) < 0.15, 0.0, r.choice([0.6, 0.7, 1.0, 1.0, 1.5], n))
    top_k = np.where(r.uniform(size=n) < 0.5, 0, r.choice([1, 20, 50, 1000], n))
    top_p = np.where(r.uniform(size=n) < 0.4, 1.0, r.choice([0.5, 0.8, 0.9, 0.95, 0.99], n))
    min_p = np.where(r.uniform(size=n) < 0.7, 0.0, r.choice([0.01, 0.05, 0.2], n))
    return temp, top_k, top_p, min_p


def _esz(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    """Each input read once (of a table the rows that occur) and each output written once."""
    c = case
    e = _esz(c["dtype"])
    if c["op"] == "embed":
        ids = _tokens(c)
        there = int((ids >= 0).sum())
        rows = len(np.unique(ids[ids >= 0]))
        if c["dir"] == "fwd":
            return {"bytes": e * c["d"] * (rows + c["tokens"]) + 4 * c["tokens"], "flops": 1.0 * c["tokens"] * c["d"]}
        out = _esz(c["grad"]) * c["d"] * (2 * rows if c["add"] else c["vocab"])
        return {"bytes": e * c["d"] * there + out + 4 * c["tokens"], "flops": 2.0 * there * c["d"]}
    if c["op"] == "norm":
        n = c["rows"] * c["d"]
        if c["dir"] == "fwd":
            return {"bytes": e * (n * (4 if c["residual"] else 2) + c["d"]), "flops": 8.0 * n}
        return {"bytes": e * (n * (4 if c["residual"] else 3) + c["d"]) + 4 * c["d"] * (2 if c["bias"] else 1),
                "flops": 14.0 * n}
    return {"bytes": e * c["rows"] * c["vocab"] + 28 * c["rows"], "flops": 20.0 * c["rows"] * c["vocab"]}


# ------------------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    rows = max(1, (1 << 26) // max(1, out[0].numel()))
    for at in range(0, shape[0], rows):
        part = out[at:at + rows]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(std).add_(mean))
    return out


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def _f32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a).astype(np.float32)).cuda()


def _embed_inputs(c, gen):
    dt, d = _dtype(c["dtype"]), c["d"]
    x = dict(ids=_i32(_tokens(c)), scale=math.sqrt(d) if c["scaled"] else 1.0)
    if c["dir"] == "fwd":
        x["table"] = _normal(gen, (c["vocab"], d), dt)
    else:
        x["grad"] = _normal(gen, (c["tokens"], d), dt, 1e-2)
        x["into"] = _normal(gen, (c["vocab"], d), _dtype(c["grad"]), 1e-2) if c["add"] else \
            torch.empty((c["vocab"], d), dtype=_dtype(c["grad"]), device="cuda")
    return x


def _norm_inputs(c, gen):
    dt, shape = _dtype(c["dtype"]), (c["rows"], c["d"])
    x = dict(x=_normal(gen, shape, dt, 1.5, 0.3), w=_normal(gen, (c["d"],), dt, 0.2, 1.0))
    x["b"] = _normal(gen, (c["d"],), dt, 0.2) if c["bias"] else None
    if c["dir"] == "bwd":
        x["dy"] = _normal(gen, shape, dt, 1e-2)
        x["dsum"] = _normal(gen, shape, dt, 1e-2) if c["residual"] else None
    else:
        x["res"] = _normal(gen, shape, dt, 1.5) if c["residual"] else None
    return x


def _sample_inputs(c, gen):
    x = dict(logits=_normal(gen, (c["rows"], c["vocab"]), _dtype(c["dtype"]), c["spread"]))
    if c["masked"]:
        hidden = torch.rand(c["vocab"], generator=gen, device="cuda") < c["masked"]
        x["logits"].masked_fill_(hidden, -math.inf)
    x["u"] = torch.rand(c["rows"], generator=gen, device="cuda")
    temp, top_k, top_p, min_p = _settings(c)
    x.update(temp=_f32(temp), top_k=None if top_k is None else _i32(top_k), top_p=_f32(top_p), min_p=_f32(min_p))
    return x


_INPUTS = {"embed": _embed_inputs, "norm": _norm_inputs, "sample": _sample_inputs}
EPS = 1e-6


class _State:
    """Inputs, output buffers, and the descriptor and workspace that a program keeps."""

    def __init__(self, c, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.c, self.x, self.plan = c, _INPUTS[c["op"]](c, gen), None
        x, dt = self.x, _dtype(c["dtype"])
        if c["op"] == "embed":
            self.out = {"out": torch.empty((c["tokens"], c["d"]), dtype=dt, device="cuda")} if c["dir"] == "fwd" else \
                {"table": x["into"]}
        elif c["op"] == "norm":
            self.out = {"out": torch.empty_like(x["x"])}
            if c["dir"] == "fwd" and c["residual"]:
                self.out["sum"] = torch.empty_like(x["x"])
            elif c["dir"] == "bwd":
                self.out["weight"] = torch.empty(c["d"], device="cuda")
                if c["bias"]:
                    self.out["bias"] = torch.empty(c["d"], device="cuda")
        else:
            self.out = {"token": torch.empty(c["rows"], dtype=torch.int32, device="cuda"),
                        "logp": torch.empty(c["rows"], device="cuda"),
                        "kept": torch.empty(c["rows"], dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    state = _State(case, seed)
    if own:
        _plan(state)
    return state


# -------------------------------------------------------------------- the library's calls
def _plan(state):
    """The descriptor and the workspace that a program sets up once."""
    from paper_2609_36246_amd import _lib as L
    c, x, need = state.c, state.x, 0
    kind = L.OLIVE_BF16 if c["dtype"] == "bf16" else L.OLIVE_F32
    if c["op"] == "embed":
        state.plan = L.make_embed_desc(c["tokens"], c["vocab"], c["d"], x["ids"], dtype=kind, scale=x["scale"])
        if c["dir"] == "bwd":
            need = L.olive_embed_workspace(state.plan)
    elif c["op"] == "norm":
        state.plan = L.make_norm_desc(c["rows"], c["d"], weight=x["w"], bias=x["b"], dtype=kind, eps=EPS,
                                      kind=L.OLIVE_NORM_LAYER if c["kind"] == "layer" else L.OLIVE_NORM_RMS)
        if c["dir"] == "bwd":
            need = L.olive_row_norm_workspace(state.plan)
    else:
        state.plan = L.make_sample_desc(c["rows"], c["vocab"], x["u"], temperature=x["temp"], top_k=x["top_k"],
                                        top_p=x["top_p"], min_p=x["min_p"], dtype=kind)
        need = L.olive_sample_workspace(state.plan)
    state.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")


def _run_own(state):
    from paper_2609_36246_amd import _lib as L
    c, x, o, p = state.c, state.x, state.out, state.plan
    if c["op"] == "embed" and c["dir"] == "fwd":
        L.olive_embed(p, x["table"], o["out"])
    elif c["op"] == "embed":
        L.olive_embed_backward(p, x["grad"], o["table"], accumulate=c["add"], workspace=state.workspace)
    elif c["op"] == "norm" and c["dir"] == "fwd":
        L.olive_row_norm(p, x["x"], o["out"], residual=x["res"], sum_out=o.get("sum"))
    elif c["op"] == "norm":
        L.olive_row_norm_backward(p, x["x"], x["dy"], o["out"], grad_sum=x["dsum"], grad_weight=o["weight"],
                                  grad_bias=o.get("bias"), workspace=state.workspace)
    else:
        L.olive_sample(p, x["logits"], o["token"], logp=o["logp"], kept=o["kept"], workspace=state.workspace)
    return o


# ------------------------------------------------------------------------ the plain forms
def _plain_embed(state):
    c, x, o = state.c, state.x, state.out
    ids = x["ids"].long()
    there = (ids >= 0)[:, None]
    at = ids.clamp(min=0)
    if c["dir"] == "fwd":
        return {"out": torch.where(there, x["table"][at].float() * x["scale"], 0.0).to(_dtype(c["dtype"]))}
    g = torch.where(there, x["grad"].float() * x["scale"], 0.0)
    into = x["into"].float() if c["add"] else torch.zeros_like(x["into"], dtype=torch.float32)
    o["table"].copy_(into.index_add_(0, at, g))
    return o


def _plain_norm(state):
    c, x = state.c, state.x
    dt, layer = _dtype(c["dtype"]), c["kind"] == "layer"
    t, w, o = x["x"].float(), x["w"].float(), {}
    if c["dir"] == "fwd" and c["residual"]:
        o["sum"] = (t + x["res"].float()).to(dt)
        t = o["sum"].float()
    if layer:
        t = t - t.mean(-1, keepdim=True)
    r = torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS)
    n = t * r
    if c["dir"] == "fwd":
        o["out"] = (n * w if x["b"] is None else n * w + x["b"].float()).to(dt)
        return o
    dy = x["dy"].float()
    o["weight"] = (dy * n).sum(0)
    if c["bias"]:
        o["bias"] = dy.sum(0)
    g = dy * w
    g = g - n * (g * n).mean(-1, keepdim=True) - (g.mean(-1, keepdim=True) if layer else 0.0)
    g = g * r
    o["out"] = (g if x["dsum"] is None else g + x["dsum"].float()).to(dt)
    return o


def _plain_sample(state):
    c, x = state.c, state.x
    z, u = x["logits"].float(), x["u"].double()[:, None]
    V = c["vocab"]
    col = lambda t, default: torch.full_like(u, default) if t is None else t.double()[:, None]  # noqa: E731
    temp, top_k, top_p, min_p = col(x["temp"], 1.0), col(x["top_k"], 0), col(x["top_p"], 1.0), col(x["min_p"], 0.0)
    greedy = temp == 0
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    w = torch.exp((z.double() - z.amax(1, keepdim=True).double()) / torch.where(greedy, 1.0, temp))
    n = (z > -math.inf).sum(1, keepdim=True)
    n = torch.where(greedy, 1, torch.where(top_k > 0, torch.minimum(n, top_k.long()), n))
    mass = torch.cumsum(torch.gather(w, 1, order), 1)
    below = mass < top_p * torch.gather(mass, 1, n - 1)
    n = torch.where(top_p < 1, torch.minimum(n, 1 + below.sum(1, keepdim=True)), n)
    n = torch.where(min_p > 0, torch.minimum(n, (w >= min_p).sum(1, keepdim=True)), n)
    at = torch.arange(V, device="cuda").expand_as(order)
    keep = torch.zeros_like(order, dtype=torch.bool).scatter_(1, order, at < n)
    mass = torch.cumsum(torch.where(keep, w, 0.0), 1)
    total = mass[:, -1:]
    token = torch.where(keep & ((mass > u * total) | (u == 0)), at, V).amin(1, keepdim=True)
    logp = torch.log(torch.gather(w, 1, token) / total)
    return {"token": token[:, 0].int(), "logp": logp[:, 0].float(), "kept": n[:, 0].int()}


_PLAIN = {"embed": _plain_embed, "norm": _plain_norm, "sample": _plain_sample}


def run(state):
    return _run_own(state) if own else _PLAIN[state.c["op"]](state)


# ---------------------------------------------------------------------------- in 64 bits
def _exact_embed(c, x):
    """Token by token where there are few, else by the rows that occur, in their order."""
    ids = torch.from_numpy(_tokens(c)).cuda()
    keep = torch.nonzero(ids >= 0)[:, 0]
    if c["dir"] == "fwd":
        out = torch.zeros((c["tokens"], c["d"]), dtype=torch.float64, device="cuda")
        out[keep] = torch.index_select(x["table"], 0, ids[keep]).double().mul_(x["scale"])
        return {"out": out}
    rows, which = torch.unique(ids[keep], return_inverse=True)
    sums = torch.zeros((len(rows), c["d"]), dtype=torch.float64, device="cuda")
    sums.index_put_((which,), x["grad"][keep].double(), accumulate=True)
    table = x["into"].double() if c["add"] else torch.zeros(x["into"].shape, dtype=torch.float64, device="cuda")
    table[rows] += x["scale"] * sums
    return {"table": table}


def _exact_norm(c, x):
    """A block of rows at a time: the layer norm's backward in its centred form."""
    o = {"out": torch.empty(x["x"].shape, dtype=torch.float64, device="cuda")}
    if c["dir"] == "fwd" and c["residual"]:
        o["sum"] = torch.empty_like(o["out"])
    w = x["w"].double()
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    for at in range(0, c["rows"], 4096):
        s = slice(at, at + 4096)
        h = x["x"][s].double()
        if "sum" in o:
            o["sum"][s] = h + x["res"][s].double()
            h = o["sum"][s].to(_dtype(c["dtype"])).double()      # what is normed is the stored sum
        h = h - h.mean(1, keepdim=True) if c["kind"] == "layer" else h
        s2 = h.pow(2).sum(1, keepdim=True) / c["d"] + EPS
        if c["dir"] == "fwd":
            o["out"][s] = h / s2.sqrt() * w + (x["b"].double() if c["bias"] else 0.0)
            continue
        dy = x["dy"][s].double()
        dw += (dy * h / s2.sqrt()).sum(0)
        db += dy.sum(0)
        g = dy * w / s2.sqrt()
        g = g - h * (g * h).sum(1, keepdim=True) / (c["d"] * s2)
        if c["kind"] == "layer":
            g = g - g.mean(1, keepdim=True)
        o["out"][s] = g + (x["dsum"][s].double() if c["residual"] else 0.0)
    if c["dir"] == "bwd":
        o["weight"] = dw
        if c["bias"]:
            o["bias"] = db
    return o


def _exact_sample(c, x):
    """Row by row, by the definition: the tokens in order, the first n of them, the draw."""
    temp, top_k, top_p, min_p = ([None] * c["rows"] if a is None else a for a in _settings(c))
    tokens, logps, kepts = [], [], []
    for i in range(c["rows"]):
        z = x["logits"][i].double()
        if temp[i] is not None and temp[i] == 0:
            tokens.append(int(torch.nonzero(z == z.max())[0]))
            logps.append(0.0)
            kepts.append(1)
            continue
        z = z / float(np.float32(1.0 if temp[i] is None else temp[i]))
        index = torch.argsort(-z, stable=True)
        p = torch.softmax(z, 0)[index]
        n = int(torch.isfinite(z).sum())
        if top_k[i]:
            n = min(n, int(top_k[i]))
        if top_p[i] is not None and top_p[i] < 1:
            share = torch.cumsum(p[:n], 0) / p[:n].sum()
            n = min(n, int(torch.searchsorted(share, float(np.float32(top_p[i])))) + 1)
        if min_p[i]:
            n = min(n, int((p >= p[0] * float(np.float32(min_p[i]))).sum()))
        among = torch.sort(index[:n]).values
        q = torch.softmax(z[among], 0)
        at = min(int(torch.searchsorted(torch.cumsum(q, 0), float(x["u"][i]), right=True)), n - 1)
        tokens.append(int(among[at]))
        logps.append(float(torch.log_softmax(z[among], 0)[at]))
        kepts.append(n)
    return {"token": torch.tensor(tokens, dtype=torch.int32), "logp": torch.tensor(logps, dtype=torch.float64),
            "kept": torch.tensor(kepts, dtype=torch.int32)}


def exact(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = _INPUTS[case["op"]](case, gen)
    return {"embed": _exact_embed, "norm": _exact_norm, "sample": _exact_sample}[case["op"]](case, x)
