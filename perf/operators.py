"""Performance cases of the block operators: what a training step runs between
the copy-out of a bucket's parameters and the copy-in of their gradients.

* ``norm`` / ``norm_bwd``       norms after and before a block, with its gate and residual scales
* ``linear`` / ``linear_bwd``   matrix product with bias, activation, factor and residual in its epilogue
* ``distill`` / ``distill_grad`` / ``distill_bwd``   distillation from a teacher's top logits: the loss, the loss
  with its gradient in one call, the gradient from a saved logsumexp

``own`` says whether ``run`` calls the framework or computes the plain form
(elementary torch operations in 32 bits).  ``exact`` computes the definition
in 64 bits.  Block sizes are those of the 8B and 70B blocks and of the toy
block; odd ones stand for ragged batches and vocabularies.
"""

from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
MAX_NORM_ELEMS = 8192 * 8192
MAX_PRODUCT = 8192 * 14336 * 4096
MAX_LOGITS = 4096 * 128256


# ------------------------------------------------------------------ cases


def _norm(name, op, tokens, hidden, dtype, stream, *, weights="block", gate_rows=1, post=True, residual=1.0, branch=1.0):
    """``dtype`` is the block's type (branch, normed output, gate), ``stream``
    the residual stream's, ``weights`` "block" or "f32"; ``gate_rows`` 0 means
    no gate, else tokens / gate_rows consecutive tokens share a row of it."""
    return {"name": name, "op": op, "tokens": tokens, "hidden": hidden, "dtype": dtype, "stream": stream,
            "weights": weights, "gate_rows": gate_rows, "post": post, "residual": residual, "branch": branch}


def _linear(name, op, m, n, k, dtype, *, act="none", bias=False, times=False, residual=False, pre=False):
    return {"name": name, "op": op, "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "bias": bias, "times": times,
            "residual": residual, "pre": pre}


def _distill(name, op, tokens, vocab, top, dtype, *, teacher="f32", tau=1.0, tail=False, holes=False):
    """``tail``: the teacher's logsumexp over its whole vocabulary is given;
    ``holes``: some rows hold fewer entries, some none."""
    return {"name": name, "op": op, "tokens": tokens, "vocab": vocab, "top": top, "dtype": dtype, "teacher": teacher,
            "tau": tau, "tail": tail, "holes": holes}


def listed():
    return [
        # One token through the norms between two blocks: the cost of a call.
        _norm("norm-1-token", "norm", 1, 4096, "bf16", "bf16"),
        # A micro-batch of the 8B block: the ordinary forward, the residual stream in 16 bits.
        _norm("norm-8b", "norm", 8192, 4096, "bf16", "bf16", residual=0.5),
        # The 70B block's backward with the stream in fp32 and a gate row for each of 8 sequences.
        _norm("norm-bwd-70b-f32-stream", "norm_bwd", 8192, 8192, "bf16", "f32", weights="f32", gate_rows=8),
        # A ragged batch of odd width in fp16, one shared gate.
        _norm("norm-bwd-ragged-f16", "norm_bwd", 1021, 771, "f16", "f16", branch=0.5),
        # One token through the 8B block's gated up projection: bound by reading the weight.
        _linear("linear-1-token", "linear", 1, 14336, 4096, "bf16", act="silu", times=True),
        # The down projection of the 8B block, added to the residual stream.
        _linear("linear-8b-down", "linear", 8192, 4096, 14336, "bf16", residual=True),
        # The gated up projection's backward: the largest step of a block.
        _linear("linear-bwd-8b-up", "linear_bwd", 4096, 14336, 4096, "bf16", act="silu", times=True),
        # Odd sizes in fp16 with a bias and GELU, the pre-activation kept for the backward.
        _linear("linear-ragged-f16", "linear", 771, 1153, 2501, "f16", act="gelu", bias=True, pre=True),
        # Training without mixed precision: the toy feed-forward's backward at a long batch.
        _linear("linear-bwd-f32", "linear_bwd", 2048, 688, 1024, "f32", act="gelu_tanh", bias=True),
        # A micro-batch's loss and gradient over the Llama 3 vocabulary.
        _distill("distill-grad-4096", "distill_grad", 4096, 128256, 64, "bf16", teacher="bf16", tau=2.0),
        # A few positions scored against a long teacher list, fp32 logits.
        _distill("distill-7-tokens-f32", "distill", 7, 32000, 256, "f32"),
        # A ragged batch over an odd vocabulary: prompts masked out, the teacher's tail mass known.
        _distill("distill-bwd-ragged-f16", "distill_bwd", 1531, 50257, 100, "f16", tau=1.5, tail=True, holes=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: one of the blocks', an odd multiple of 8, or any."""
    kind = rng.random()
    if kind < 0.4:
        return rng.choice([w for w in (256, 688, 1024, 1792, 4096, 8192, 14336, 28672) if lo <= w <= hi])
    n = _log_int(rng, lo, hi)
    return n // 16 * 16 + 8 if kind < 0.7 else n | 1


def draw(rng):
    """One more case: sizes log-uniform over the listed ranges, every
    direction, type and option."""
    op = rng.choice(["norm", "norm_bwd", "linear", "linear", "linear_bwd", "linear_bwd", "distill", "distill_grad",
                     "distill_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        if op.startswith("norm"):
            tokens, hidden = _log_int(rng, 1, 16384), min(_width(rng, 64, 14336), 14336)
            if tokens * hidden > MAX_NORM_ELEMS:
                continue
            gate_rows = rng.choice([0, 1, 1] + [g for g in (2, 8, tokens) if tokens % g == 0])
            case = _norm("", op, tokens, hidden, dtype, rng.choice([dtype, "f32"]), weights=rng.choice(["block", "f32"]),
                         gate_rows=gate_rows, post=rng.random() < 0.7, residual=rng.choice([1.0, 0.75]),
                         branch=rng.choice([1.0, 0.25]))
        elif op.startswith("linear"):
            m, n, k = _log_int(rng, 1, 8192), _width(rng, 64, 28672), _width(rng, 64, 28672)
            products = 1 if op == "linear" else 2
            if m * n * k * products * (4 if dtype == "f32" else 1) > MAX_PRODUCT or n * k > 1 << 28:
                continue
            act = rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"])
            case = _linear("", op, m, n, k, dtype, act=act, bias=rng.random() < 0.5, times=rng.random() < 0.4,
                           residual=op == "linear" and rng.random() < 0.5, pre=op == "linear" and rng.random() < 0.3)
        else:
            tokens, vocab = _log_int(rng, 1, 8192), _log_int(rng, 1000, 128256)
            if tokens * vocab * (2 if dtype == "f32" else 1) > MAX_LOGITS:
                continue
            case = _distill("", op, tokens, vocab, _log_int(rng, 1, 512), dtype, teacher=rng.choice(["bf16", "f16", "f32"]),
                            tau=rng.choice([1.0, 2.0, 0.7]), tail=rng.random() < 0.3, holes=rng.random() < 0.5)
        del case["name"]
        return case


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape, dtype, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(scale).add_(shift).to(dtype)

    op = case["op"]
    if op.startswith("norm"):
        t, h = case["tokens"], case["hidden"]
        stream, block = DTYPES[case["stream"]], DTYPES[case["dtype"]]
        weights = torch.float32 if case["weights"] == "f32" else block
        s = {"case": case, "branch": normal(t, h, dtype=block),
             "pre_weight": normal(h, dtype=weights, scale=0.1, shift=1.0),
             "post_weight": normal(h, dtype=weights, scale=0.1, shift=1.0) if case["post"] else None,
             "gate": normal(case["gate_rows"], h, dtype=block, scale=0.5) if case["gate_rows"] else None}
        if op == "norm":
            s |= {"x": normal(t, h, dtype=stream, scale=3.0), "y": torch.empty(t, h, dtype=stream, device=DEVICE),
                  "h": torch.empty(t, h, dtype=block, device=DEVICE)}
        else:
            s |= {"y": normal(t, h, dtype=stream, scale=3.0), "dy": normal(t, h, dtype=stream, scale=1e-2),
                  "dh": normal(t, h, dtype=block, scale=1e-2), "dx": torch.empty(t, h, dtype=stream, device=DEVICE),
                  "dbranch": torch.empty(t, h, dtype=block, device=DEVICE)}
            for w in ("pre_weight", "post_weight", "gate"):
                s["d" + w] = None if s[w] is None else torch.empty_like(s[w])
        return s
    if op.startswith("linear"):
        m, n, k, dtype = case["m"], case["n"], case["k"], DTYPES[case["dtype"]]
        s = {"case": case, "x": normal(m, k, dtype=dtype), "weight": normal(n, k, dtype=dtype, scale=k ** -0.5),
             "times": normal(m, n, dtype=dtype) if case["times"] else None}
        if op == "linear":
            s |= {"bias": normal(n, dtype=dtype, scale=0.1) if case["bias"] else None,
                  "residual": normal(m, n, dtype=dtype) if case["residual"] else None,
                  "out": torch.empty(m, n, dtype=dtype, device=DEVICE),
                  "pre": torch.empty(m, n, dtype=dtype, device=DEVICE) if case["pre"] else None}
        else:
            kept = case["act"] != "none" or case["times"]
            s |= {"dout": normal(m, n, dtype=dtype, scale=1e-2), "pre": normal(m, n, dtype=dtype) if kept else None,
                  "dx": torch.empty(m, k, dtype=dtype, device=DEVICE), "dweight": torch.empty(n, k, dtype=dtype, device=DEVICE),
                  "dbias": torch.empty(n, dtype=dtype, device=DEVICE) if case["bias"] else None,
                  "dtimes": torch.empty(m, n, dtype=dtype, device=DEVICE) if case["times"] else None}
        return s
    t, v, k, dtype = case["tokens"], case["vocab"], case["top"], DTYPES[case["dtype"]]
    logits = normal(t, v, dtype=dtype, scale=2.5)
    # The teacher agrees with the student in part; its top entries are those of its whole row.
    whole = logits.float().mul_(0.8).add_(torch.randn(t, v, generator=g, device=DEVICE))
    top, ids = whole.topk(k, dim=1)
    s = {"case": case, "logits": logits, "teacher": top.to(DTYPES[case["teacher"]]), "ids": ids.to(torch.int32),
         "teacher_lse": torch.logsumexp(whole.div_(case["tau"]), 1) if case["tail"] else None,
         "loss": torch.empty(t, device=DEVICE)}
    del whole
    if case["holes"]:
        held = torch.randint(0, k + 1, (t, 1), generator=g, device=DEVICE)
        held[torch.rand(t, 1, generator=g, device=DEVICE) < 0.5] = k
        held[torch.rand(t, 1, generator=g, device=DEVICE) < 0.2] = 0
        s["ids"][torch.arange(k, device=DEVICE)[None] >= held] = -1
    if op != "distill":
        # A mean over the batch; in fp16 under the loss scale that its small gradients need.
        s["dloss"] = torch.rand(t, generator=g, device=DEVICE).add_(0.5).mul_((8192 if dtype is torch.float16 else 1) / t)
        s["dlogits"] = torch.empty_like(logits)
    if op == "distill_bwd":
        s["lse"] = torch.logsumexp(logits.float() / case["tau"], 1)
    return s


def work(case):
    op = case["op"]
    if op.startswith("norm"):
        t, h, b, st = case["tokens"], case["hidden"], BYTES[case["dtype"]], BYTES[case["stream"]]
        wide = (b if case["weights"] == "block" else 4) * h * (2 if case["post"] else 1) + b * h * case["gate_rows"]
        if op == "norm":
            return {"bytes": t * h * (2 * st + 2 * b) + wide, "flops": 12 * t * h}
        return {"bytes": t * h * (3 * st + 3 * b) + 2 * wide, "flops": 30 * t * h}
    if op.startswith("linear"):
        m, n, k, b = case["m"], case["n"], case["k"], BYTES[case["dtype"]]
        kept = 1 if case["act"] != "none" or case["times"] else 0
        if op == "linear":
            extra = m * n * (case["times"] + case["residual"] + case["pre"]) + n * case["bias"]
            return {"bytes": b * (m * k + n * k + m * n + extra), "flops": 2 * m * n * k}
        extra = m * n * (kept + 2 * case["times"]) + n * case["bias"]
        return {"bytes": b * (2 * m * k + 2 * n * k + m * n + extra), "flops": 4 * m * n * k}
    t, v, k, b = case["tokens"], case["vocab"], case["top"], BYTES[case["dtype"]]
    rows = t * k * (BYTES[case["teacher"]] + 4) + 4 * t * (1 + case["tail"])
    if op == "distill":
        return {"bytes": t * v * b + rows, "flops": 4 * t * v}
    return {"bytes": 2 * t * v * b + rows + 4 * t, "flops": 8 * t * v}


# ------------------------------------------------------------------ one pass


def run(s):
    return _framework(s) if own else _plain(s)


def _framework(s):
    import paper_2411_00284_amd as fw

    case, op = s["case"], s["case"]["op"]
    if op == "norm":
        fw.block_norm(s["x"], branch=s["branch"], pre_weight=s["pre_weight"], post_weight=s["post_weight"], gate=s["gate"],
                      y=s["y"], h=s["h"], residual_scale=case["residual"], branch_scale=case["branch"], eps=EPS)
        return {"y": s["y"], "h": s["h"]}
    if op == "norm_bwd":
        fw.block_norm_backward(s["y"], dy=s["dy"], dh=s["dh"], branch=s["branch"], pre_weight=s["pre_weight"],
                               post_weight=s["post_weight"], gate=s["gate"], dx=s["dx"], dbranch=s["dbranch"],
                               dpre_weight=s["dpre_weight"], dpost_weight=s["dpost_weight"], dgate=s["dgate"],
                               residual_scale=case["residual"], branch_scale=case["branch"], eps=EPS)
        return {k: s[k] for k in ("dx", "dbranch", "dpre_weight", "dpost_weight", "dgate")}
    if op == "linear":
        fw.linear(s["x"], s["weight"], s["out"], bias=s["bias"], activation=case["act"], times=s["times"],
                  residual=s["residual"], pre=s["pre"])
        return {"out": s["out"], "pre": s["pre"]}
    if op == "linear_bwd":
        fw.linear_backward(s["dout"], s["x"], s["weight"], activation=case["act"], pre=s["pre"], times=s["times"],
                           dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"], dtimes=s["dtimes"])
        return {k: s[k] for k in ("dx", "dweight", "dbias", "dtimes")}
    if op == "distill":
        fw.distill_loss(s["logits"], s["teacher"], s["ids"], s["loss"], temperature=case["tau"],
                        teacher_lse=s["teacher_lse"])
        return {"loss": s["loss"]}
    if op == "distill_grad":
        fw.distill_loss(s["logits"], s["teacher"], s["ids"], s["loss"], temperature=case["tau"],
                        teacher_lse=s["teacher_lse"], dloss=s["dloss"], dlogits=s["dlogits"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    fw.distill_loss_backward(s["dloss"], s["logits"], s["teacher"], s["ids"], s["lse"], s["dlogits"],
                             temperature=case["tau"], teacher_lse=s["teacher_lse"])
    return {"dlogits": s["dlogits"]}


def _f32(t):
    return None if t is None else t.float()


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "norm":
        return _plain_norm(s, case)
    if op == "norm_bwd":
        return _plain_norm_bwd(s, case)
    if op == "linear":
        z = s["x"].float() @ s["weight"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        out = _act(z, case["act"])
        if s["times"] is not None:
            out = out * s["times"].float()
        if s["residual"] is not None:
            out = out + s["residual"].float()
        dtype = s["x"].dtype
        return {"out": out.to(dtype), "pre": None if s["pre"] is None else z.to(dtype)}
    if op == "linear_bwd":
        dout, pre, times, dtype = s["dout"].float(), _f32(s["pre"]), _f32(s["times"]), s["x"].dtype
        dz, dtimes = dout, None
        if times is not None:
            dtimes = (dout * _act(pre, case["act"])).to(dtype)
            dz = dz * times
        if case["act"] != "none":
            dz = dz * _act_slope(pre, case["act"])
        return {"dx": (dz @ s["weight"].float()).to(dtype), "dweight": (dz.t() @ s["x"].float()).to(dtype),
                "dbias": dz.sum(0).to(dtype) if s["dbias"] is not None else None, "dtimes": dtimes}
    return _plain_distill(s, case)


def _unit(v):
    """(v / rms(v), 1 / rms(v)) of every row."""
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _rows_of(gate, tokens):
    return gate.float().repeat_interleave(tokens // gate.shape[0], 0) if gate.shape[0] > 1 else gate.float()


def _plain_norm(s, case):
    x, b = s["x"].float(), s["branch"].float()
    if s["post_weight"] is not None:
        b = _unit(b)[0] * s["post_weight"].float()
    if s["gate"] is not None:
        b = b * _rows_of(s["gate"], case["tokens"])
    y = case["residual"] * x + case["branch"] * b
    h = _unit(y)[0] * s["pre_weight"].float()
    return {"y": y.to(s["x"].dtype), "h": h.to(s["branch"].dtype)}


def _plain_norm_bwd(s, case):
    t, n = case["tokens"], case["hidden"]
    y, b, dh = s["y"].float(), s["branch"].float(), s["dh"].float()
    u, r = _unit(y)
    du = dh * s["pre_weight"].float()
    gy = s["dy"].float() + r * (du - u * (du * u).mean(1, keepdim=True))
    got = {"dx": (case["residual"] * gy).to(s["dx"].dtype),
           "dpre_weight": (dh * u).sum(0).to(s["pre_weight"].dtype), "dpost_weight": None, "dgate": None}
    dn, normed = case["branch"] * gy, b
    if s["post_weight"] is not None:
        ub, rb = _unit(b)
        normed = ub * s["post_weight"].float()
    if s["gate"] is not None:
        rows = s["gate"].shape[0]
        got["dgate"] = (dn * normed).reshape(rows, t // rows, n).sum(1).to(s["gate"].dtype)
        dn = dn * _rows_of(s["gate"], t)
    if s["post_weight"] is not None:
        got["dpost_weight"] = (dn * ub).sum(0).to(s["post_weight"].dtype)
        dn = dn * s["post_weight"].float()
        dn = rb * (dn - ub * (dn * ub).mean(1, keepdim=True))
    got["dbranch"] = dn.to(s["branch"].dtype)
    return got


def _act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    w = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + w) + 0.5 * z * (1 - w * w) * c * (1 + 3 * 0.044715 * z * z)


def _plain_distill(s, case):
    tau, ids, op = case["tau"], s["ids"].long(), case["op"]
    valid = ids >= 0
    at = ids.clamp(min=0)
    u = s["logits"].float() / tau
    v = (s["teacher"].float() / tau).masked_fill(~valid, -math.inf)
    live = valid.any(1)
    if s["teacher_lse"] is None:
        top = v.max(1, keepdim=True).values.masked_fill(~live[:, None], 0.0)
        total = top + torch.exp(v - top).sum(1, keepdim=True).log()
        total = total.masked_fill(~live[:, None], 0.0)
    else:
        total = s["teacher_lse"][:, None]
    p = torch.exp(v - total)
    if op == "distill_bwd":
        lse = s["lse"][:, None]
    else:
        top = u.max(1, keepdim=True).values
        lse = top + torch.exp(u - top).sum(1, keepdim=True).log()
    got = {}
    if op != "distill_bwd":
        terms = p * ((v - total) - (u.gather(1, at) - lse))
        got["loss"] = tau * tau * terms.masked_fill(~valid, 0.0).sum(1)
    if op != "distill":
        g = (torch.exp(u - lse) * p.sum(1, keepdim=True)).scatter_add_(1, at, -p)
        got["dlogits"] = (g * (tau * s["dloss"])[:, None]).to(s["logits"].dtype)
    return got


# ------------------------------------------------------------------ the definition in 64 bits


def exact(case, seed):
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in prepare(case, seed).items()
         if k not in ("h", "dx", "out", "dlogits", "dweight", "loss", "dbranch", "dtimes")}
    op = case["op"]
    if op.startswith("norm"):
        t, n = case["tokens"], case["hidden"]
        post, gate = s["post_weight"], s["gate"]
        full = torch.ones(1, n, dtype=torch.float64, device=DEVICE) if gate is None else gate
        full = full.unsqueeze(1).expand(full.shape[0], t // full.shape[0], n).reshape(t, n)
        b = s["branch"]
        rb = b.pow(2).mean(1).add(EPS).pow(-0.5).unsqueeze(1)
        normed = b if post is None else b * rb * post
        if op == "norm":
            y = case["residual"] * s["x"] + case["branch"] * full * normed
            return {"y": y, "h": y * y.pow(2).mean(1).add(EPS).pow(-0.5).unsqueeze(1) * s["pre_weight"]}
        y, w = s["y"], s["pre_weight"]
        r = y.pow(2).mean(1).add(EPS).pow(-0.5).unsqueeze(1)
        inner = (s["dh"] * w * y).mean(1).unsqueeze(1)
        gy = s["dy"] + s["dh"] * w * r - y * r.pow(3) * inner
        dn = case["branch"] * full * gy
        out = {"dx": case["residual"] * gy, "dpre_weight": (s["dh"] * y * r).sum(0), "dbranch": dn, "dpost_weight": None,
               "dgate": None}
        if post is not None:
            out["dpost_weight"] = (dn * b * rb).sum(0)
            out["dbranch"] = dn * post * rb - b * rb.pow(3) * (dn * post * b).mean(1).unsqueeze(1)
        if gate is not None:
            out["dgate"] = (case["branch"] * gy * normed).unflatten(0, (gate.shape[0], -1)).sum(1)
        return out
    if op.startswith("linear"):
        act = case["act"]
        if op == "linear":
            z = torch.mm(s["x"], s["weight"].t().contiguous())
            z = z if s["bias"] is None else z + s["bias"]
            out = _curve(z, act)[0]
            out = out if s["times"] is None else out * s["times"]
            return {"out": out if s["residual"] is None else out + s["residual"], "pre": z if case["pre"] else None}
        value, slope = (None, 1.0) if s["pre"] is None else _curve(s["pre"], act)
        dz = s["dout"] * slope if s["times"] is None else s["dout"] * s["times"] * slope
        return {"dx": torch.mm(dz, s["weight"]), "dweight": torch.mm(dz.t().contiguous(), s["x"]),
                "dbias": dz.sum(0) if case["bias"] else None,
                "dtimes": s["dout"] * value if case["times"] else None}
    tau, ids = case["tau"], s["ids"]
    t, v = s["logits"].shape
    held = ids >= 0
    score = torch.where(held, s["teacher"] / tau, -math.inf)
    norm = torch.logsumexp(score, 1) if s["teacher_lse"] is None else s["teacher_lse"]
    logp = torch.where(held, score - norm[:, None], -math.inf)
    p = torch.where(held, logp.exp(), 0.0)
    lse = s["lse"] if op == "distill_bwd" else torch.logsumexp(s["logits"] / tau, 1)
    logq = (s["logits"] / tau).sub_(lse[:, None])
    got = {}
    if op != "distill_bwd":
        picked = logq.gather(1, torch.where(held, ids, 0).long())
        got["loss"] = tau ** 2 * torch.where(held, p * (logp - picked), 0.0).sum(1)
    if op != "distill":
        dense = torch.zeros(t, v, dtype=torch.float64, device=DEVICE)
        dense.scatter_add_(1, torch.where(held, ids, 0).long(), p)
        got["dlogits"] = logq.exp_().mul_(p.sum(1, keepdim=True)).sub_(dense).mul_((s["dloss"] * tau)[:, None])
    return got


def _curve(z, act):
    """Value and slope of the activation."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.relu(z), (z > 0).double()
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * (-z * z / 2).exp() / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    arg = a * (z + 0.044715 * z ** 3)
    cdf = torch.sigmoid(2 * arg)
    return z * cdf, cdf + z * 2 * cdf * (1 - cdf) * a * (1 + 0.134145 * z ** 2)
