"""The operators of a residual block over the cells of a grid, or over tokens, and of the end of its training step, as cases
that can be timed and compared.

Kinds of pass (`op`):
  linear         y = act(x W^T + b) + residual, for training with x W^T + b beside it
  linear_bwd     gradients of x, W and b for a given gradient of y and the kept x W^T + b
  block_norm     the norm behind a block, its gate, the residual sum and the norm before the next block
  block_norm_bwd its gradients for given gradients of the sum and of the normed sum
  clip           the norm of all gradients of a step together, and the gradients brought under a largest norm

`own` selects the library's entry points; without it the same formulas run as elementary torch operations in 32 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS_NORM, _EPS_CLIP = 1e-5, 1e-6


def _named(name, case):
    return {**({"name": name} if name else {}), **case}


def _linear(op, p, k, n, act="none", dtype="f32", bias=True, residual=False, keep=False, name=None):
    return _named(name, {"op": op, "p": p, "k": k, "n": n, "act": act, "dtype": dtype, "bias": bias,
                         "residual": residual, "keep": keep})


def _norm(op, n, p, c, kind="rms", h="f32", f=None, post=False, gate="channel", alpha=1.0, name=None):
    return _named(name, {"op": op, "n": n, "p": p, "c": c, "kind": kind, "h": h, "f": f or h, "post": post, "gate": gate,
                         "alpha": alpha})


def _clip(tensors, dtype="f32", part=0.25, name=None):
    return _named(name, {"op": "clip", "tensors": tensors, "dtype": dtype, "part": part})


def listed():
    return [
        # one token through the first product of a block of width 512 at work: the call itself counts
        _linear("linear", 1, 512, 2048, act="gelu", dtype="bf16", name="token_linear"),
        # odd sizes throughout, behind a low level of a network over several scenes
        _linear("linear", 3 * 37 * 41 * 29, 72, 97, act="silu", dtype="f16", residual=True, name="odd_linear"),
        # channels widened over the grid of the paper's experiments
        _linear("linear", 160 ** 3, 32, 64, act="silu", name="voxel160_linear"),
        # a batch of 64 scenes with 1024 tokens each through a block of width 512, in training
        _linear("linear", 65536, 512, 2048, act="gelu", dtype="bf16", keep=True, name="width512_linear"),
        # the same batch, gradients
        _linear("linear_bwd", 65536, 512, 2048, act="gelu", dtype="bf16", name="width512_linear_bwd"),
        # the cells of 8 scenes' triplanes (24 planes) as tokens of a small network, gradients
        _linear("linear_bwd", 24 * 256 * 256, 32, 128, act="gelu", dtype="bf16", name="planes256_linear_bwd"),
        # one token behind its block at work
        _norm("block_norm", 1, 1, 512, h="bf16", post=True, name="token_block_norm"),
        # odd sizes throughout
        _norm("block_norm", 3, 37 * 41 * 29, 72, kind="layer", h="f16", gate="sample", alpha=0.7, name="odd_block_norm"),
        # the cells of 8 scenes' triplanes: sums in fp32, blocks in bf16, a gate for each plane
        _norm("block_norm_bwd", 24, 256 * 256, 32, kind="layer", h="f32", f="bf16", gate="sample", name="planes256_block_norm_bwd"),
        # 64 scenes of 1024 tokens of width 512
        _norm("block_norm_bwd", 64, 1024, 512, h="bf16", post=True, name="width512_block_norm_bwd"),
        # a small decoder's gradients, each step of fitting a scene: launches count
        _clip("64x16+64+64x64+64+4x64+4", name="decoder_clip"),
        # the gradients of a grid, of the matrices of 6 layers of width 512 and of their vectors
        _clip("4096000x32+24*512x512+6*2048x512+6*512x2048+12*512+6*2048", name="network_clip"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_linear(rng):
    op = rng.choice(["linear", "linear", "linear_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    k, n = (_log_int(rng, 3, 2048) if rng.random() < 0.4 else rng.choice([16, 32, 64, 72, 128, 256, 512, 1024, 2048]) for _ in range(2))
    products, values = 65536 * 512 * 2048 // (1 if dtype != "f32" else 4), 160 ** 3 * 96 // (1 if op == "linear" else 2)
    top = min(products // (k * n), values // (k + n))
    p = rng.randint(1, 16) if op == "linear" and rng.random() < 0.25 else _log_int(rng, min(64, top), top)
    return _linear(op, p, k, n, act=rng.choice(["none", "relu", "silu", "gelu", "gelu"]), dtype=dtype,
                   bias=rng.random() < 0.8, residual=op == "linear" and rng.random() < 0.4,
                   keep=op == "linear" and rng.random() < 0.4)


def _draw_norm(rng):
    op = rng.choice(["block_norm", "block_norm_bwd"])
    c = _log_int(rng, 4, 4096) if rng.random() < 0.4 else rng.choice([16, 32, 64, 72, 128, 256, 512, 1024, 2048])
    n = rng.choice([1, 1, 2, 3, 8, 24, 64])
    top = 24 * 256 * 256 * 32 // (n * c)
    h = rng.choice(["f32", "bf16", "f16"])
    return _norm(op, n, _log_int(rng, 1, max(2, top)), c, kind=rng.choice(["rms", "layer"]), h=h,
                 f=rng.choice([h, "bf16"]) if h == "f32" else h, post=rng.random() < 0.5,
                 gate=rng.choice(["none", "channel", "sample"]), alpha=rng.choice([1.0, 1.0, 0.7]))


def _draw_clip(rng):
    terms, left = [], 1 << 27
    for _ in range(rng.randint(1, 12)):
        rows, cols, count = _log_int(rng, 1, 1 << 21), _log_int(rng, 1, 2100), rng.choice([1, 1, 1, 2, 3, 5])
        if rows * cols * count <= left:
            terms.append("%d*%dx%d" % (count, rows, cols))
            left -= rows * cols * count
    return _clip("+".join(terms) or "513", dtype=rng.choice(["f32", "f32", "bf16", "f16"]), part=rng.choice([0.1, 0.5, 3.0]))


def draw(rng):
    return rng.choice([_draw_linear, _draw_linear, _draw_norm, _draw_norm, _draw_clip])(rng)


def _sizes(case):
    """Numbers of values of the tensors of a text of terms: sizes rows x cols or rows, each with a count in front where there are several."""
    out = []
    for term in case["tensors"].split("+"):
        count, _, shape = term.rpartition("*")
        out += [math.prod(int(v) for v in shape.split("x"))] * int(count or 1)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    state = dict(case)
    if case["op"].startswith("linear"):
        p, k, n, dtype = case["p"], case["k"], case["n"], _TYPES[case["dtype"]]
        state["x"] = rand(p, k).to(dtype)
        state["weight"] = (rand(n, k) / math.sqrt(k)).to(dtype)
        state["b"] = 0.2 * rand(n) if case["bias"] else None
        state["res"] = rand(p, n).to(dtype) if case["residual"] else None
        if case["op"] == "linear_bwd":
            state["d_y"] = (1e-2 * rand(p, n)).to(dtype)
            # what the forward kept
            state["pre"] = None if case["act"] == "none" else _pre(state).to(dtype)
        return state
    if case["op"].startswith("block_norm"):
        n, p, c = case["n"], case["p"], case["c"]
        h, f = _TYPES[case["h"]], _TYPES[case["f"]]
        # the sum over the blocks so far has some strong channels, a block's result does not
        state["in"] = (rand(n, p, c) * (0.5 + 3 * torch.rand(c, device="cuda", generator=gen).pow(4)) + 0.3 * rand(c)).to(h)
        state["block"] = (0.6 * rand(n, p, c) + 0.1).to(f)
        state["gamma"], state["beta"] = 1 + 0.2 * rand(c), 0.2 * rand(c) if case["kind"] == "layer" else None
        state["post_gamma"] = 1 + 0.2 * rand(c) if case["post"] else None
        state["g"] = {"none": None, "channel": 0.5 + 0.2 * rand(c), "sample": 0.5 + 0.2 * rand(n, c)}[case["gate"]]
        if case["op"] == "block_norm_bwd":
            state["d_sum"], state["d_y"] = (1e-2 * rand(n, p, c)).to(h), (1e-2 * rand(n, p, c)).to(f)
        return state
    sizes = _sizes(case)
    # gradients of tensors differ by orders of magnitude; those in fp16 are of a loss that was scaled up
    scales = [10.0 ** (i % 4) * (1e-2 if case["dtype"] == "f16" else 1e-3 / math.sqrt(s)) for i, s in enumerate(sizes)]
    state["grads"] = [rand(s).mul_(v).to(_TYPES[case["dtype"]]) for s, v in zip(sizes, scales)]
    state["outs"] = [torch.empty_like(g) for g in state["grads"]]
    state["max_norm"] = case["part"] * math.sqrt(sum(s * v * v for s, v in zip(sizes, scales)))
    return state


# ---- plain forms -----------------------------------------------------------------------------------------------

def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2.0)))
    return z.clamp(min=0) if act == "relu" else z


def _act_slope(z, act):
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return (z > 0).to(z.dtype)


def _pre(s):
    z = s["x"].float() @ s["weight"].float().t()
    return z if s["b"] is None else z + s["b"]


def _plain_linear(s):
    dtype = s["x"].dtype
    z = _pre(s)
    y = _act(z, s["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    out = {"y": y.to(dtype)}
    if s["keep"]:
        out["pre"] = z.to(dtype)
    return out


def _plain_linear_bwd(s):
    d_z = s["d_y"].float()
    if s["pre"] is not None:
        d_z = d_z * _act_slope(s["pre"].float(), s["act"])
    out = {"d_x": (d_z @ s["weight"].float()).to(s["x"].dtype), "d_weight": d_z.t() @ s["x"].float()}
    if s["b"] is not None:
        out["d_bias"] = d_z.sum(0)
    return out


def _normed(x, kind):
    """The normed rows and what they were multiplied by."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS_NORM)
    return x * rstd, rstd


def _normed_grad(d, xh, rstd, kind):
    d = d - xh * (d * xh).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if kind == "layer" else 0)
    return d * rstd


def _gate(s):
    return None if s["g"] is None else s["g"].view(-1, 1, s["c"])


def _plain_block_norm(s):
    h, f = s["in"].float(), s["block"].float()
    u = _normed(f, s["kind"])[0] * s["post_gamma"] if s["post"] else f
    gate = _gate(s)
    total = s["alpha"] * h + (u if gate is None else gate * u)
    y = _normed(total, s["kind"])[0] * s["gamma"]
    if s["beta"] is not None:
        y = y + s["beta"]
    return {"sum": total.to(s["in"].dtype), "y": y.to(s["block"].dtype)}


def _plain_block_norm_bwd(s):
    kind, gate = s["kind"], _gate(s)
    h, f, d_y = s["in"].float(), s["block"].float(), s["d_y"].float()
    fh, f_rstd = _normed(f, kind) if s["post"] else (f, None)
    u = fh * s["post_gamma"] if s["post"] else fh
    xh, rstd = _normed(s["alpha"] * h + (u if gate is None else gate * u), kind)
    g = s["d_sum"].float() + _normed_grad(d_y * s["gamma"], xh, rstd, kind)
    d_u = g if gate is None else gate * g
    out = {"d_h": (s["alpha"] * g).to(s["in"].dtype), "d_gamma": (d_y * xh).sum((0, 1))}
    if s["post"]:
        out["d_post_gamma"] = (d_u * fh).sum((0, 1))
        d_u = _normed_grad(d_u * s["post_gamma"], fh, f_rstd, kind)
    out["d_f"] = d_u.to(s["block"].dtype)
    if s["beta"] is not None:
        out["d_beta"] = d_y.sum((0, 1))
    if gate is not None:
        out["d_gate"] = (g * u).sum(1) if s["g"].dim() == 2 else (g * u).sum((0, 1))
    return out


def _plain_clip(s):
    # (sums of the tensors in 32 bits, as torch adds them up, the few of them together in 64)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).double().sum().sqrt().float()
    factor = (s["max_norm"] / (norm + _EPS_CLIP)).clamp(max=1.0)
    return {"norm": norm, "outs": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ---- the library's entry points --------------------------------------------------------------------------------

def _lin(s, lp):
    act = {"none": lp.LP_ACT_NONE, "relu": lp.LP_ACT_RELU, "silu": lp.LP_ACT_SILU, "gelu": lp.LP_ACT_GELU}[s["act"]]
    return lp.Linear(s["weight"], s["b"], act)


def _own_linear(s):
    import paper_2404_19760_amd as lp
    y, pre = lp.linear_fwd(_lin(s, lp), s["x"], residual=s["res"], keep=s["keep"])
    return {"y": y, "pre": pre} if s["keep"] else {"y": y}


def _own_linear_bwd(s):
    import paper_2404_19760_amd as lp
    d_x, d_weight, d_bias = lp.linear_bwd(_lin(s, lp), s["x"], s["pre"], s["d_y"])
    return {"d_x": d_x, "d_weight": d_weight, **({} if s["b"] is None else {"d_bias": d_bias})}


def _block(s, lp):
    return lp.ResidualNorm(lp.LP_NORM_LAYER if s["kind"] == "layer" else lp.LP_NORM_RMS, s["gamma"], s["beta"], s["post"],
                           s["post_gamma"], s["g"], s["alpha"], _EPS_NORM)


def _own_block_norm(s):
    import paper_2404_19760_amd as lp
    total, y = lp.residual_norm_fwd(_block(s, lp), s["in"], s["block"])
    return {"sum": total, "y": y}


def _own_block_norm_bwd(s):
    import paper_2404_19760_amd as lp
    d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate = lp.residual_norm_bwd(_block(s, lp), s["in"], s["block"], s["d_sum"], s["d_y"])
    out = {"d_h": d_h, "d_gamma": d_gamma, "d_post_gamma": d_post_gamma, "d_f": d_f, "d_beta": d_beta, "d_gate": d_gate}
    return {k: v for k, v in out.items() if v is not None}


def _own_clip(s):
    import paper_2404_19760_amd as lp
    return {"norm": lp.clip_grad_norm(s["grads"], s["max_norm"], _EPS_CLIP, outs=s["outs"]), "outs": s["outs"]}


_PLAIN = {"linear": _plain_linear, "linear_bwd": _plain_linear_bwd, "block_norm": _plain_block_norm,
          "block_norm_bwd": _plain_block_norm_bwd, "clip": _plain_clip}
_OWN = {"linear": _own_linear, "linear_bwd": _own_linear_bwd, "block_norm": _own_block_norm,
        "block_norm_bwd": _own_block_norm_bwd, "clip": _own_clip}


def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


def work(case):
    if case["op"].startswith("linear"):
        p, k, n = case["p"], case["k"], case["n"]
        size = _BYTES[case["dtype"]]
        if case["op"] == "linear":
            moved = size * p * (k + n * (1 + case["residual"] + case["keep"])) + size * n * k
            return {"bytes": moved, "flops": 2 * p * k * n}
        return {"bytes": size * p * (2 * k + n * (1 if case["act"] == "none" else 2)) + (size + 4) * n * k, "flops": 4 * p * k * n}
    if case["op"].startswith("block_norm"):
        values = case["n"] * case["p"] * case["c"]
        h, f = _BYTES[case["h"]], _BYTES[case["f"]]
        return {"bytes": values * (2 * h + 2 * f), "flops": 10 * values} if case["op"] == "block_norm" else \
            {"bytes": values * (3 * h + 3 * f), "flops": 30 * values}
    values = sum(_sizes(case))
    # each gradient in and out once: what the chip does not hold between the sum and the scaling is read twice
    return {"bytes": 2 * _BYTES[case["dtype"]] * values, "flops": 3 * values}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _exact_act(z, act):
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return {"silu": torch.nn.functional.silu, "relu": torch.relu, "none": lambda t: 1.0 * t}[act](z)


def _exact_linear(s):
    z = torch.nn.functional.linear(s["x"].double(), s["weight"].double(), None if s["b"] is None else s["b"].double())
    y = _exact_act(z, s["act"])
    if s["res"] is not None:
        y += s["res"]
    return {"y": y, "pre": z} if s["keep"] else {"y": y}


def _exact_linear_bwd(s):
    d_z = s["d_y"].double()
    if s["pre"] is not None:
        z = s["pre"].double().requires_grad_(True)
        d_z, = torch.autograd.grad(_exact_act(z, s["act"]), z, d_z)
    d_weight = torch.zeros(s["n"], s["k"], dtype=torch.float64, device="cuda")
    for rows in range(0, s["p"], 1 << 18):
        d_weight += d_z[rows:rows + (1 << 18)].t().contiguous() @ s["x"][rows:rows + (1 << 18)].double()
    out = {"d_x": torch.mm(d_z, s["weight"].double()), "d_weight": d_weight}
    return out if s["b"] is None else {**out, "d_bias": torch.ones(1, s["p"], dtype=torch.float64, device="cuda").mm(d_z)[0]}


def _exact_rows(x, kind):
    if kind == "layer":
        return torch.nn.functional.layer_norm(x, x.shape[-1:], eps=_EPS_NORM)
    return x * (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + _EPS_NORM).rsqrt()


def _exact_block_norm(s):
    names = ["in", "block", "gamma", "beta", "post_gamma", "g"]
    back = s["op"] == "block_norm_bwd"
    t = {k: None if s[k] is None else s[k].double().requires_grad_(back) for k in names}
    u = t["block"] if not s["post"] else t["post_gamma"] * _exact_rows(t["block"], s["kind"])
    if s["g"] is not None:
        u = u * (t["g"] if s["g"].dim() == 1 else t["g"].unsqueeze(1))
    total = torch.add(u, t["in"], alpha=s["alpha"])
    y = _exact_rows(total, s["kind"]) * t["gamma"]
    if t["beta"] is not None:
        y = y + t["beta"]
    if not back:
        return {"sum": total, "y": y}
    leaves = [k for k in names if t[k] is not None]
    grads = dict(zip(leaves, torch.autograd.grad([total, y], [t[k] for k in leaves], [s["d_sum"].double(), s["d_y"].double()])))
    result = {"d_h": "in", "d_gamma": "gamma", "d_post_gamma": "post_gamma", "d_f": "block", "d_beta": "beta", "d_gate": "g"}
    return {k: grads[v] for k, v in result.items() if v in grads}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(s)
    if case["op"] == "linear_bwd":
        return _exact_linear_bwd(s)
    if case["op"].startswith("block_norm"):
        return _exact_block_norm(s)
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + _EPS_CLIP))
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "outs": [g.double() * factor for g in s["grads"]]}
