"""Performance cases of the gated feed-forward, of activations kept in 8 bits,
and of the policy loss.

* ``gated`` / ``gated_bwd``   both projections of a gated feed-forward, their activation and product; the
  gradient, from projections kept in the type or in 8 bits, which also writes the product again
* ``checkpoint``   a matrix to 8 bits and back: what a step does in its forward and in its backward pass
* ``saved_bwd``    a linear layer's gradient from an input and a pre-activation kept in 8 bits
* ``policy`` / ``policy_grad`` / ``policy_bwd``   clipped policy loss with its KL term over a vocabulary: the
  loss, the loss with its gradient in one call, the gradient from a saved logsumexp

``own`` says whether ``run`` calls the framework or computes the plain form
(elementary torch operations in 32 bits).  ``exact`` computes the definition
in 64 bits.  Sizes are those of the 8B block and of the toy block; odd ones
stand for ragged batches and vocabularies.
"""

from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GROUP = 32                         # neighbouring columns that share a scale
SAVED_BYTES = 1 + 1 / GROUP
MAX_PRODUCT = 2 * 8192 * 14336 * 4096
MAX_ELEMS = 8192 * 14336
MAX_LOGITS = 4096 * 128256


# ------------------------------------------------------------------ cases


def _gated(name, op, m, n, k, dtype, *, act="silu", kept="none", saved_x=False):
    """``kept``: how the two projections are kept for the gradient: "none",
    "type" (the case's own) or "8bit"; ``saved_x``: x too is kept in 8 bits."""
    return {"name": name, "op": op, "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "kept": kept, "saved_x": saved_x}


def _checkpoint(name, rows, cols, dtype):
    return {"name": name, "op": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype}


def _saved(name, m, n, k, dtype, *, act="none", bias=False):
    return {"name": name, "op": "saved_bwd", "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "bias": bias}


def _policy(name, op, tokens, vocab, dtype, *, kl=0.0, low=0.2, high=0.2, tau=1.0, prompt=False):
    """``kl``: the KL term's weight (0: no reference policy); ``prompt``: some
    tokens are prompt or padding and count for nothing."""
    return {"name": name, "op": op, "tokens": tokens, "vocab": vocab, "dtype": dtype, "kl": kl, "low": low, "high": high,
            "tau": tau, "prompt": prompt}


def listed():
    return [
        # One token through the 8B block's feed-forward: bound by reading both weights.
        _gated("gated-1-token", "gated", 1, 14336, 4096, "bf16"),
        # A long prompt, or a forward pass that will be computed again: nothing is kept.
        _gated("gated-8b", "gated", 8192, 14336, 4096, "bf16"),
        # A training forward that keeps both projections in 8 bits, read back here to be compared.
        _gated("gated-8b-saved", "gated", 2048, 14336, 4096, "bf16", kept="8bit"),
        # The 8B block's largest backward step, everything it reads again kept in 8 bits.
        _gated("gated-bwd-8b-saved", "gated_bwd", 4096, 14336, 4096, "bf16", kept="8bit", saved_x=True),
        # Odd sizes in fp16 with GELU, the projections kept as they are.
        _gated("gated-ragged-f16", "gated", 771, 1153, 2501, "f16", act="gelu", kept="type"),
        # Training without mixed precision: the toy feed-forward's backward at a long batch.
        _gated("gated-bwd-f32", "gated_bwd", 2048, 688, 1024, "f32", kept="type"),
        # One token's activations: the cost of a call.
        _checkpoint("checkpoint-1-token", 1, 4096, "bf16"),
        # A micro-batch of the 8B block's residual stream.
        _checkpoint("checkpoint-8b", 8192, 4096, "bf16"),
        # A GELU layer's backward in fp16 whose input and pre-activation were kept in 8 bits.
        _saved("linear-bwd-saved-f16", 2048, 14336, 4096, "f16", act="gelu", bias=True),
        # A micro-batch's policy loss and gradient over the Llama 3 vocabulary.
        _policy("policy-grad-4096", "policy_grad", 4096, 128256, "bf16", kl=0.05),
        # A few sampled tokens scored, fp32 logits.
        _policy("policy-7-tokens-f32", "policy", 7, 32000, "f32", kl=0.1),
        # A ragged batch over an odd vocabulary: prompts masked out, a wider upper clip, sampled at a temperature.
        _policy("policy-bwd-ragged-f16", "policy_bwd", 1531, 50257, "f16", kl=0.02, high=0.28, tau=0.9, prompt=True),
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
    op = rng.choice(["gated", "gated", "gated", "gated_bwd", "gated_bwd", "checkpoint", "saved_bwd", "policy", "policy_grad",
                     "policy_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    act = rng.choice(["none", "relu", "silu", "silu", "gelu", "gelu_tanh"])
    while True:
        if op in ("gated", "gated_bwd", "saved_bwd"):
            m, n, k = _log_int(rng, 1, 8192), _width(rng, 64, 28672), _width(rng, 64, 28672)
            products = 4 if op == "gated_bwd" else 2
            if m * n * k * products * (4 if dtype == "f32" else 1) > MAX_PRODUCT or n * k > 1 << 27:
                continue
            if op == "saved_bwd":
                case = _saved("", m, n, k, dtype, act=act, bias=rng.random() < 0.5)
            elif op == "gated":
                # fp32 projections are kept as they are.
                case = _gated("", op, m, n, k, dtype, act=act, kept=rng.choice(["none", "type", "type" if dtype == "f32" else "8bit"]))
            else:
                case = _gated("", op, m, n, k, dtype, act=act, kept=rng.choice(["type", "8bit"]), saved_x=rng.random() < 0.5)
        elif op == "checkpoint":
            rows, cols = _log_int(rng, 1, 32768), _width(rng, 64, 28672)
            if rows * cols > MAX_ELEMS:
                continue
            case = _checkpoint("", rows, cols, dtype)
        else:
            tokens, vocab = _log_int(rng, 1, 8192), _log_int(rng, 1000, 128256)
            if tokens * vocab * (2 if dtype == "f32" else 1) > MAX_LOGITS:
                continue
            case = _policy("", op, tokens, vocab, dtype, kl=rng.choice([0.0, 0.05, 0.2]), low=rng.choice([0.2, 0.1]),
                           high=rng.choice([0.2, 0.28]), tau=rng.choice([1.0, 0.8, 1.2]), prompt=rng.random() < 0.5)
        del case["name"]
        return case


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape, dtype, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(scale).to(dtype)

    def empty(*shape, dtype):
        return torch.empty(*shape, dtype=dtype, device=DEVICE)

    def saved_like(rows, cols):
        """The buffers of a matrix in 8 bits: its codes, and a scale's exponent for each group of columns."""
        return empty(rows, cols, dtype=torch.int8), empty(rows, -(-cols // GROUP), dtype=torch.uint8)

    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = {"case": case}
    if op in ("gated", "gated_bwd"):
        m, n, k = case["m"], case["n"], case["k"]
        x = normal(m, k, dtype=dtype)
        s |= {"gate_weight": normal(n, k, dtype=dtype, scale=k ** -0.5), "up_weight": normal(n, k, dtype=dtype, scale=k ** -0.5),
              "out": empty(m, n, dtype=dtype)}
        if op == "gated":
            s["x"] = x
            s |= {"gate": saved_like(m, n), "up": saved_like(m, n)} if case["kept"] == "8bit" else {}
            if case["kept"] != "none":          # as they are, or what 8 bits are read back into
                s |= {"gate_values": empty(m, n, dtype=dtype), "up_values": empty(m, n, dtype=dtype)}
            return s
        gate, up = normal(m, n, dtype=dtype), normal(m, n, dtype=dtype)
        s |= {"x": _to_8bit(x) if case["saved_x"] else x, "gate": _to_8bit(gate) if case["kept"] == "8bit" else gate,
              "up": _to_8bit(up) if case["kept"] == "8bit" else up, "dout": normal(m, n, dtype=dtype, scale=1e-2),
              "dx": empty(m, k, dtype=dtype), "dgate_weight": empty(n, k, dtype=dtype), "dup_weight": empty(n, k, dtype=dtype)}
        return s
    if op == "checkpoint":
        rows, cols = case["rows"], case["cols"]
        x = torch.randn(rows, cols, generator=g, device=DEVICE)
        # A stream has a few columns that are much larger than the others.
        x[:, torch.randint(0, cols, (max(1, cols // 256),), generator=g, device=DEVICE)] *= 20.0
        return s | {"x": x.to(dtype), "saved": saved_like(rows, cols), "out": empty(rows, cols, dtype=dtype)}
    if op == "saved_bwd":
        m, n, k = case["m"], case["n"], case["k"]
        return s | {"x": _to_8bit(normal(m, k, dtype=dtype)), "weight": normal(n, k, dtype=dtype, scale=k ** -0.5),
                    "pre": _to_8bit(normal(m, n, dtype=dtype)) if case["act"] != "none" else None,
                    "dout": normal(m, n, dtype=dtype, scale=1e-2), "dx": empty(m, k, dtype=dtype),
                    "dweight": empty(n, k, dtype=dtype), "dbias": empty(n, dtype=dtype) if case["bias"] else None}
    t, v, tau = case["tokens"], case["vocab"], case["tau"]
    logits = normal(t, v, dtype=dtype, scale=2.5)
    # Sampled actions are mostly likely ones: the best of a few at random.
    few = torch.randint(0, v, (t, 64), generator=g, device=DEVICE)
    actions = few.gather(1, logits.gather(1, few).argmax(1, keepdim=True))
    lse = _row_lse(logits, tau)
    now = logits.gather(1, actions)[:, 0].float() / tau - lse
    s |= {"logits": logits, "actions": actions[:, 0].to(torch.int32),
          "old_logp": now + normal(t, dtype=torch.float32, scale=0.15), "advantages": normal(t, dtype=torch.float32),
          "ref_logp": now + normal(t, dtype=torch.float32, scale=0.3) if case["kl"] else None}
    if case["prompt"]:
        s["actions"][torch.rand(t, generator=g, device=DEVICE) < 0.3] = -1
    if op != "policy_bwd":
        s |= {"loss": empty(t, dtype=torch.float32), "logp": empty(t, dtype=torch.float32)}
    if op != "policy":
        # A mean over the batch; in fp16 under the loss scale that its small gradients need.
        s["dloss"] = torch.rand(t, generator=g, device=DEVICE).add_(0.5).mul_((8192 if dtype is torch.float16 else 1) / t)
        s["dlogits"] = torch.empty_like(logits)
    if op == "policy_bwd":
        s["lse"] = lse
    return s


def _row_lse(logits, tau):
    """The logsumexp of logits / tau, a part of the rows at a time."""
    step = max(1, (1 << 27) // logits.shape[1])
    return torch.cat([torch.logsumexp(rows.float() / tau, 1) for rows in logits.split(step)])


def work(case):
    op, b = case["op"], BYTES[case["dtype"]]
    if op in ("gated", "gated_bwd"):
        m, n, k = case["m"], case["n"], case["k"]
        kept = {"none": 0, "type": b, "8bit": SAVED_BYTES}[case["kept"]]
        if op == "gated":
            back = 2 * m * n * (SAVED_BYTES + b) if case["kept"] == "8bit" else 0
            return {"bytes": b * (m * k + 2 * n * k + m * n) + 2 * kept * m * n + back, "flops": 4 * m * n * k}
        x = SAVED_BYTES if case["saved_x"] else b
        return {"bytes": b * (4 * n * k + m * k + 2 * m * n) + x * m * k + 2 * kept * m * n, "flops": 8 * m * n * k}
    if op == "checkpoint":
        return {"bytes": 2 * case["rows"] * case["cols"] * (b + SAVED_BYTES), "flops": 8 * case["rows"] * case["cols"]}
    if op == "saved_bwd":
        m, n, k = case["m"], case["n"], case["k"]
        pre = SAVED_BYTES if case["act"] != "none" else 0
        return {"bytes": b * (2 * n * k + m * k + m * n + n * case["bias"]) + SAVED_BYTES * m * k + pre * m * n,
                "flops": 4 * m * n * k}
    t, v = case["tokens"], case["vocab"]
    rows = 4 * t * (3 + (case["kl"] != 0))
    if op == "policy":
        return {"bytes": t * v * b + rows + 8 * t, "flops": 4 * t * v}
    return {"bytes": 2 * t * v * b + rows + 4 * t, "flops": 8 * t * v}


# ------------------------------------------------------------------ one pass


def run(s):
    return _framework(s) if own else _plain(s)


def _framework(s):
    import paper_2411_00284_amd as fw

    case, op = s["case"], s["case"]["op"]

    def held(v):
        return fw.Checkpoint(*v) if isinstance(v, tuple) else v

    if op == "gated":
        keep = {}
        if case["kept"] == "8bit":
            keep = {"gate": held(s["gate"]), "up": held(s["up"])}
        elif case["kept"] == "type":
            keep = {"gate": s["gate_values"], "up": s["up_values"]}
        fw.gated_linear(s["x"], s["gate_weight"], s["up_weight"], s["out"], activation=case["act"], **keep)
        if case["kept"] == "none":
            return {"out": s["out"]}
        if case["kept"] == "8bit":
            fw.checkpoint_restore(keep["gate"], s["gate_values"])
            fw.checkpoint_restore(keep["up"], s["up_values"])
        return {"out": s["out"], "gate": s["gate_values"], "up": s["up_values"]}
    if op == "gated_bwd":
        fw.gated_linear_backward(s["dout"], held(s["x"]), s["gate_weight"], s["up_weight"], held(s["gate"]), held(s["up"]),
                                 activation=case["act"], out=s["out"], dx=s["dx"], dgate_weight=s["dgate_weight"],
                                 dup_weight=s["dup_weight"])
        return {k: s[k] for k in ("out", "dx", "dgate_weight", "dup_weight")}
    if op == "checkpoint":
        saved = held(s["saved"])
        fw.checkpoint_save(s["x"], saved)
        fw.checkpoint_restore(saved, s["out"])
        return {"out": s["out"]}
    if op == "saved_bwd":
        fw.linear_backward(s["dout"], held(s["x"]), s["weight"], activation=case["act"], pre=held(s["pre"]), dx=s["dx"],
                           dweight=s["dweight"], dbias=s["dbias"])
        return {k: s[k] for k in ("dx", "dweight", "dbias")}
    options = {"ref_logp": s["ref_logp"], "clip_low": case["low"], "clip_high": case["high"], "kl_weight": case["kl"],
               "temperature": case["tau"]}
    if op == "policy_bwd":
        fw.policy_loss_backward(s["dloss"], s["logits"], s["actions"], s["old_logp"], s["advantages"], s["lse"], s["dlogits"],
                                **options)
        return {"dlogits": s["dlogits"]}
    grad = {"dloss": s["dloss"], "dlogits": s["dlogits"]} if op == "policy_grad" else {}
    fw.policy_loss(s["logits"], s["actions"], s["old_logp"], s["advantages"], s["loss"], s["logp"], **options, **grad)
    return {"loss": s["loss"], "logp": s["logp"], "dlogits": grad.get("dlogits")}


def _to_8bit(x):
    """Codes and scale exponents of a matrix.  A group's scale is the least
    power of two with which its largest value rounds to at most 127; a group
    that holds a value that is not finite stands for NaN (exponent byte 255)."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -cols % GROUP)).reshape(rows, -1, GROUP)
    most = v.abs().amax(2)
    mantissa, exponent = torch.frexp(most)                       # most = mantissa 2^exponent, mantissa in [1/2, 1)
    exponent = (exponent - 7 + (mantissa >= 127.5 / 128).int()).clamp(min=-126)
    exponent = torch.where(most == 0, -126, exponent)
    codes = torch.round(torch.ldexp(v, -exponent.unsqueeze(2)))
    fine = torch.isfinite(most)
    codes = torch.where(fine.unsqueeze(2), codes, 0.0).to(torch.int8).reshape(rows, -1)[:, :cols]
    return codes.contiguous(), torch.where(fine, exponent + 127, 255).to(torch.uint8)


def _from_8bit(saved):
    codes, scales = saved
    rows, cols = codes.shape
    scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    scale = torch.where(scales == 255, math.nan, scale)
    return codes.float() * scale.repeat_interleave(GROUP, 1)[:, :cols]


def _held_f32(v):
    return None if v is None else _from_8bit(v) if isinstance(v, tuple) else v.float()


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    dtype = DTYPES[case["dtype"]]
    if op == "gated":
        x = s["x"].float()
        g, u = x @ s["gate_weight"].float().t(), x @ s["up_weight"].float().t()
        got = {"out": (_act(g, case["act"]) * u).to(dtype)}
        if case["kept"] != "none":
            got |= {"gate": _kept(g, case["kept"], dtype), "up": _kept(u, case["kept"], dtype)}
        return got
    if op == "gated_bwd":
        dout, x, g, u = s["dout"].float(), _held_f32(s["x"]), _held_f32(s["gate"]), _held_f32(s["up"])
        value = _act(g, case["act"])
        dg, du = dout * u * _act_slope(g, case["act"]), dout * value
        return {"out": (value * u).to(dtype), "dx": (dg @ s["gate_weight"].float() + du @ s["up_weight"].float()).to(dtype),
                "dgate_weight": (dg.t() @ x).to(dtype), "dup_weight": (du.t() @ x).to(dtype)}
    if op == "checkpoint":
        return {"out": _from_8bit(_to_8bit(s["x"])).to(dtype)}
    if op == "saved_bwd":
        dz, x, z = s["dout"].float(), _held_f32(s["x"]), _held_f32(s["pre"])
        if z is not None:
            dz = dz * _act_slope(z, case["act"])
        return {"dx": (dz @ s["weight"].float()).to(dtype), "dweight": (dz.t() @ x).to(dtype),
                "dbias": None if s["dbias"] is None else dz.sum(0).to(dtype)}
    return _plain_policy(s, case)


def _kept(z, how, dtype):
    return _from_8bit(_to_8bit(z)).to(dtype) if how == "8bit" else z.to(dtype)


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
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        w = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + w) + 0.5 * z * (1 - w * w) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain_policy(s, case):
    tau, op, actions = case["tau"], case["op"], s["actions"].long()
    live, at = actions >= 0, actions.clamp(min=0)[:, None]
    u = s["logits"].float() / tau
    if op == "policy_bwd":
        lse = s["lse"][:, None]
    else:
        top = u.max(1, keepdim=True).values
        lse = top + torch.exp(u - top).sum(1, keepdim=True).log()
    # A token's few values in 64 bits: the KL term is a small difference, and the clip a border.
    logp = (u.gather(1, at).double() - lse.double())[:, 0]
    ratio = torch.exp(logp - s["old_logp"].double())
    a = s["advantages"].double()
    clipped = ratio.clamp(1 - case["low"], 1 + case["high"])
    loss, slope = -torch.minimum(ratio * a, clipped * a), torch.where(ratio * a <= clipped * a, -ratio * a, 0.0)
    if case["kl"]:
        d = s["ref_logp"].double() - logp
        loss, slope = loss + case["kl"] * (torch.exp(d) - d - 1), slope + case["kl"] * (1 - torch.exp(d))
    got = {}
    if op != "policy_bwd":
        got = {"loss": loss.masked_fill(~live, 0.0).float(), "logp": logp.masked_fill(~live, 0.0).float(), "dlogits": None}
    if op != "policy":
        weight = (s["dloss"].double() * slope / tau).masked_fill(~live, 0.0).float()[:, None]
        q = torch.exp(u - lse)
        got["dlogits"] = (q * -weight).scatter_add_(1, at, weight).to(s["logits"].dtype)
    return got


# ------------------------------------------------------------------ the definition in 64 bits


def exact(case, seed):
    s, op, act = prepare(case, seed), case["op"], case.get("act")

    def wide(v):
        if not isinstance(v, tuple):
            return None if v is None else v.double()
        codes, scales = v
        column = torch.arange(codes.shape[1], device=DEVICE) // GROUP
        power = scales.double() - 127
        return codes.double() * torch.exp2(power)[:, column]

    if op == "gated":
        x = wide(s["x"])
        g = torch.mm(x, wide(s["gate_weight"]).t().contiguous())
        u = torch.mm(x, wide(s["up_weight"]).t().contiguous())
        got = {"out": _curve(g, act)[0] * u}
        if case["kept"] != "none":
            got |= {"gate": _near(g) if case["kept"] == "8bit" else g, "up": _near(u) if case["kept"] == "8bit" else u}
        return got
    if op == "gated_bwd":
        dout, x, g, u = wide(s["dout"]), wide(s["x"]), wide(s["gate"]), wide(s["up"])
        value, slope = _curve(g, act)
        dg, du = dout * slope * u, dout * value
        return {"out": value * u, "dx": torch.mm(dg, wide(s["gate_weight"])) + torch.mm(du, wide(s["up_weight"])),
                "dgate_weight": torch.mm(dg.t().contiguous(), x), "dup_weight": torch.mm(du.t().contiguous(), x)}
    if op == "checkpoint":
        return {"out": _near(s["x"].double())}
    if op == "saved_bwd":
        dz = wide(s["dout"])
        if s["pre"] is not None:
            dz = dz * _curve(wide(s["pre"]), act)[1]
        return {"dx": torch.mm(dz, wide(s["weight"])), "dweight": torch.mm(dz.t().contiguous(), wide(s["x"])),
                "dbias": dz.sum(0) if case["bias"] else None}
    tau, t = case["tau"], case["tokens"]
    live = s["actions"] >= 0
    row, action = torch.arange(t, device=DEVICE), torch.where(live, s["actions"], 0).long()
    logq = s["logits"].double().div_(tau)
    logq -= (s["lse"].double() if op == "policy_bwd" else torch.logsumexp(logq, 1))[:, None]
    logp, adv = logq[row, action], s["advantages"].double()
    ratio = (logp - s["old_logp"].double()).exp()
    low, high = 1 - case["low"], 1 + case["high"]
    # Where raising the ratio would go on gaining past the clip, the objective is flat.
    flat = ((adv > 0) & (ratio > high)) | ((adv < 0) & (ratio < low))
    loss = -adv * torch.where(flat, torch.where(adv > 0, high, low).double(), ratio)
    slope = torch.where(flat, 0.0, -adv * ratio)
    if case["kl"]:
        gap = s["ref_logp"].double() - logp
        loss, slope = loss + case["kl"] * (torch.expm1(gap) - gap), slope - case["kl"] * torch.expm1(gap)
    got = {}
    if op != "policy_bwd":
        got = {"loss": torch.where(live, loss, 0.0), "logp": torch.where(live, logp, 0.0), "dlogits": None}
    if op != "policy":
        each = torch.where(live, s["dloss"].double() * slope / tau, 0.0)
        dlogits = logq.exp_().mul_(-each[:, None])
        dlogits[row, action] += each
        got["dlogits"] = dlogits
    return got


def _near(v):
    """The values that 8 bits hold: multiples, up to 127, of the power of two that fits a group."""
    rows, cols = v.shape
    column = torch.arange(-(-cols // GROUP) * GROUP, device=DEVICE).clamp(max=cols - 1)
    groups = v[:, column].unflatten(1, (-1, GROUP))
    step = torch.exp2(torch.floor(torch.log2(groups.abs().amax(2, keepdim=True).clamp(min=2.0 ** -120))) - 6)
    step = torch.where((groups / step).abs().amax(2, keepdim=True) >= 127.5, step * 2, step)
    return ((groups / step).round() * step).flatten(1)[:, :cols]


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
    cdf = torch.sigmoid(2 * a * (z + 0.044715 * z ** 3))
    return z * cdf, cdf + z * 2 * cdf * (1 - cdf) * a * (1 + 0.134145 * z ** 2)
