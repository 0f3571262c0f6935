"""The operators that stand next to the Renderer and the Splatter when a network over a grid is trained, as cases
that can be timed and compared: group norm with an activation over channel-last grids, and the orthogonalised
(Newton-Schulz) update of weight matrices.

Kinds of pass (`op`):
  norm        group norm + activation, forward alone (a trained network at work)
  norm_train  forward and, for a given gradient of its output, backward
  orth        orthogonalisation of a list of matrices
  muon        one optimiser step over a list of weight matrices: momentum, orthogonalisation, update

A list of matrices is a text of terms rows x cols, each with a count in front where several of one shape lie in one tensor:
"8*64x32+64x64".  `own` selects the library's entry points; without it the same formulas run as elementary torch
operations in 32 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_COEFFS = (3.4445, -4.775, 2.0315)
_STEPS, _EPS_ORTH, _EPS_NORM = 5, 1e-7, 1e-5
_LR, _MU, _DECAY = 0.02, 0.95, 0.01


def _norm(op, n, p, channels, groups, act="silu", x="f32", y=None, occupied=0.0, name=None):
    return {**({"name": name} if name else {}), "op": op, "n": n, "p": p, "channels": channels, "groups": groups, "act": act, "x": x,
            "y": y or x, "occupied": occupied}


def _mats(op, mats, dtype="f32", nesterov=True, name=None):
    return {**({"name": name} if name else {}), "op": op, "mats": mats, "dtype": dtype, "nesterov": nesterov}


def listed():
    return [
        # one plane of the smallest triplane, shown as a preview: the call itself counts
        _norm("norm", 1, 32 * 32, 16, 4, name="plane32_norm"),
        # a splatted 64^3 grid, statistics over the cells that something landed in, in training
        _norm("norm_train", 1, 64 ** 3, 32, 8, occupied=0.2, name="splat64_norm_train"),
        # odd sizes throughout: a low level of a network over several scenes, channels that fill no power of two
        _norm("norm_train", 3, 37 * 41 * 29, 72, 6, act="gelu", x="f16", name="odd_norm_train"),
        # a batch of 8 scenes' triplanes (24 planes) in bf16, a reconstruction network in training
        _norm("norm_train", 24, 256 * 256, 32, 8, x="bf16", name="planes256_norm_train"),
        # the grid of the paper's experiments, in training
        _norm("norm_train", 1, 160 ** 3, 32, 8, name="voxel160_norm_train"),
        # the finest voxel grid, on its way to a Renderer that reads it in bf16
        _norm("norm", 1, 256 ** 3, 16, 4, x="f32", y="bf16", name="voxel256_norm"),
        # the matrices of one small decoder MLP, each step of fitting a scene: launches count
        _mats("muon", "64x16+64x64+4x64", name="decoder_muon"),
        # the decoders of 64 scenes fitted side by side
        _mats("muon", "64*64x32+64*64x64+64*4x64", nesterov=False, name="scenes64_muon"),
        # convolution weights of a network over a grid (3x3x3 kernels), gradients in bf16
        _mats("orth", "2*64x864+2*64x1728+2*128x1728+2*128x3456+2*256x6912", dtype="bf16", name="conv_orth"),
        # single matrices of odd sizes, tall and wide
        _mats("orth", "333x1001+1000x257+97x61", name="odd_orth"),
        # the matrices of a transformer of 6 layers of width 512
        _mats("muon", "24*512x512+6*2048x512+6*512x2048", name="width512_muon"),
        # few large matrices
        _mats("orth", "2*2048x2048+1024x4096", name="large_orth"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_train", "norm_train", "orth", "muon"])
    if op.startswith("norm"):
        groups = rng.choice([1, 2, 4, 8, 16])
        channels = groups * rng.choice([1, 2, 3, 4, 8, 12, 16]) if rng.random() < 0.5 else max(groups, rng.choice([16, 32, 64]))
        x = rng.choice(["f32", "f32", "bf16", "f16"])
        n = rng.choice([1, 1, 2, 3, 8, 24])
        p = max(64, _log_int(rng, 1024, 1 << 26) // (n * channels))
        # (a gradient at the kink of a ReLU hangs on the last bit of its argument: forward alone)
        act = rng.choice(["silu", "silu", "gelu", "none", "relu" if op == "norm" else "silu"])
        return _norm(op, n, p, channels, groups, act=act, x=x,
                     y="bf16" if x == "f32" and rng.random() < 0.25 else x, occupied=rng.choice([0.0, 0.0, 0.05, 0.3]))
    terms, left = [], 2.8e11   # operations of a step's products, under the largest listed case's
    for _ in range(rng.randint(1, 4)):
        rows, cols = _log_int(rng, 4, 2100), _log_int(rng, 16, 2100)
        m, n = min(rows, cols), max(rows, cols)
        while 5 * (4.0 * m * m * n + 2.0 * m ** 3) > left / 4:
            rows, cols, m, n = rows // 2 + 1, cols // 2 + 1, m // 2 + 1, n // 2 + 1
        terms.append("%d*%dx%d" % (rng.choice([1, 1, 2, 3, 8, 31]) if max(m, n) < 300 else rng.choice([1, 1, 2]), rows, cols))
    return _mats(op, "+".join(terms), dtype="f32" if op == "muon" else rng.choice(["f32", "f32", "bf16", "f16"]), nesterov=rng.random() < 0.7)


def _shapes(case):
    out = []
    for term in case["mats"].split("+"):
        count, _, shape = term.rpartition("*")
        rows, cols = shape.split("x")
        out.append((int(count or 1), int(rows), int(cols)))
    return out


def _gradient(count, rows, cols, gen):
    """A gradient of a weight matrix: few strong directions above noise of every direction."""
    rank = max(1, min(rows, cols) // 8)
    left = torch.randn(count, rows, rank, device="cuda", generator=gen)
    right = torch.randn(count, rank, cols, device="cuda", generator=gen)
    return 1e-3 * (left @ right / math.sqrt(rank) + 0.1 * torch.randn(count, rows, cols, device="cuda", generator=gen))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    state = dict(case)
    if case["op"].startswith("norm"):
        n, p, c = case["n"], case["p"], case["channels"]
        x = rand(n, p, c).mul_(0.7).add_(0.5 * rand(c))
        if case["occupied"]:
            # the weight sums a Splatter leaves: whole runs of cells that nothing landed in hold zeros
            runs = torch.rand(n, -(-p // 16), device="cuda", generator=gen) < case["occupied"]
            weight = torch.rand(n, p, device="cuda", generator=gen) * runs.repeat_interleave(16, 1)[:, :p]
            state["weight"] = weight.contiguous()
            x.mul_((weight > 0).unsqueeze(-1))
        state["in"] = x.to(_TYPES[case["x"]])
        del x
        state["gamma"], state["beta"] = 1 + 0.2 * rand(c), 0.2 * rand(c)
        if case["op"] == "norm_train":
            state["dy"] = (1e-2 * rand(n, p, c)).to(_TYPES[case["y"]])
        return state
    grads = [_gradient(*s, gen) for s in _shapes(case)]
    if case["op"] == "orth":
        state["in"] = [g.to(_TYPES[case["dtype"]]) for g in grads]
        return state
    state["grads"] = grads
    state["momenta"] = [5 * _gradient(*s, gen) for s in _shapes(case)]
    state["weights"] = [rand(*s) * math.sqrt(2.0 / s[2]) for s in _shapes(case)]
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
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _plain_norm(s):
    n, p, c, groups = s["n"], s["p"], s["channels"], s["groups"]
    split = lambda t: t.view(n, p, groups, c // groups)  # noqa: E731
    x = split(s["in"].float())
    gamma, beta = s["gamma"].view(groups, -1), s["beta"].view(groups, -1)
    if s["occupied"]:
        on = (s["weight"] > 0).view(n, p, 1, 1)
        count = (on.sum(1, keepdim=True) * (c // groups)).clamp(min=1)
        keep = lambda t: torch.where(on, t, torch.zeros((), device=t.device))  # noqa: E731
    else:
        count, keep = p * (c // groups), lambda t: t  # noqa: E731
    mean = keep(x).sum((1, 3), keepdim=True) / count
    rstd = 1 / torch.sqrt(keep((x - mean).square()).sum((1, 3), keepdim=True) / count + _EPS_NORM)
    xh = (x - mean) * rstd
    z = xh * gamma + beta
    y = keep(_act(z, s["act"])).view(n, p, c).to(_TYPES[s["y"]])
    if s["op"] == "norm":
        return {"y": y}
    g = keep(split(s["dy"].float()) * _act_slope(z, s["act"]))
    d_gamma, d_beta = keep(g * xh).sum((0, 1)).view(c), g.sum((0, 1)).view(c)
    gg = g * gamma
    d_x = rstd * (gg - (gg.sum((1, 3), keepdim=True) + xh * keep(gg * xh).sum((1, 3), keepdim=True)) / count)
    return {"y": y, "d_x": keep(d_x).view(n, p, c).to(s["in"].dtype), "d_gamma": d_gamma, "d_beta": d_beta}


def _plain_orth(g):
    x = g.float()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-2, -1).contiguous()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + _EPS_ORTH)
    a, b, c = _COEFFS
    for _ in range(_STEPS):
        gram = x @ x.transpose(-2, -1).contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(-2, -1).contiguous() if tall else x


def _plain_muon(w, g, m, nesterov):
    m.mul_(_MU).add_(g)
    o = _plain_orth(g + _MU * m if nesterov else m)
    w.mul_(1 - _LR * _DECAY).sub_(o, alpha=_LR * math.sqrt(max(1.0, w.shape[-2] / w.shape[-1])))


# ---- the library's entry points --------------------------------------------------------------------------------

def _own_norm(s):
    import paper_2404_19760_amd as lp
    act = {"none": lp.LP_ACT_NONE, "relu": lp.LP_ACT_RELU, "silu": lp.LP_ACT_SILU, "gelu": lp.LP_ACT_GELU}[s["act"]]
    norm = lp.GroupNorm(s["groups"], s["gamma"], s["beta"], act, _EPS_NORM, s.get("weight"))
    y, stats = lp.group_norm_fwd(norm, s["in"], _TYPES[s["y"]])
    if s["op"] == "norm":
        return {"y": y}
    d_x, d_gamma, d_beta = lp.group_norm_bwd(norm, s["in"], stats, s["dy"])
    return {"y": y, "d_x": d_x, "d_gamma": d_gamma, "d_beta": d_beta}


def _own_orth(s):
    import paper_2404_19760_amd as lp
    return {"out": lp.orthogonalize(s["in"], steps=_STEPS, eps=_EPS_ORTH)}


def _own_muon(s):
    import paper_2404_19760_amd as lp
    lp.muon_step(s["weights"], s["grads"], s["momenta"], lr=_LR, momentum=_MU, nesterov=s["nesterov"], weight_decay=_DECAY,
                 scale=lp.LP_MUON_SCALE_ASPECT, steps=_STEPS, eps=_EPS_ORTH)


def run(state):
    if state["op"].startswith("norm"):
        return _own_norm(state) if own else _plain_norm(state)
    if state["op"] == "orth":
        return _own_orth(state) if own else {"out": [_plain_orth(g).to(g.dtype) for g in state["in"]]}
    if own:
        _own_muon(state)
    else:
        for w, g, m in zip(state["weights"], state["grads"], state["momenta"]):
            _plain_muon(w, g, m, state["nesterov"])
    return {"weights": state["weights"], "momenta": state["momenta"]}


def work(case):
    if case["op"].startswith("norm"):
        cells = case["n"] * case["p"]
        values = cells * case["channels"]
        moved = values * (_BYTES[case["x"]] + _BYTES[case["y"]]) + (4 * cells if case["occupied"] else 0)
        if case["op"] == "norm":
            return {"bytes": moved, "flops": 10 * values}
        return {"bytes": moved + values * (2 * _BYTES[case["x"]] + _BYTES[case["y"]]) + (4 * cells if case["occupied"] else 0), "flops": 30 * values}
    values = flops = 0
    for count, rows, cols in _shapes(case):
        m, n = min(rows, cols), max(rows, cols)
        values += count * m * n
        # the two symmetric products need half their entries only
        flops += count * _STEPS * (3.0 * m * m * n + 1.0 * m ** 3)
    return {"bytes": values * (2 * _BYTES[case["dtype"]] if case["op"] == "orth" else 20), "flops": flops}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _exact_norm(s):
    n, c, groups = s["n"], s["channels"], s["groups"]
    size = c // groups
    gamma, beta = s["gamma"].double(), s["beta"].double()
    y, d_x = torch.zeros_like(s["in"], dtype=torch.float64), torch.zeros_like(s["in"], dtype=torch.float64)
    d_gamma, d_beta = torch.zeros_like(gamma), torch.zeros_like(beta)
    for i in range(n):
        on = (s["weight"][i] > 0).nonzero()[:, 0] if s["occupied"] else torch.arange(s["p"], device="cuda")
        if not len(on):
            continue
        for j in range(groups):
            span = slice(j * size, (j + 1) * size)
            x = s["in"][i, :, span][on].double()
            var, mean = torch.var_mean(x, correction=0)
            rstd = (var + _EPS_NORM).rsqrt()
            xh = (x - mean) * rstd
            z = torch.addcmul(beta[span], xh, gamma[span]).requires_grad_(True)
            out = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu, "none": lambda t: 1.0 * t}[s["act"]](z)
            y[i, on, span] = out.detach()
            if s["op"] == "norm_train":
                dz, = torch.autograd.grad(out, z, s["dy"][i, :, span][on].double())
                d_gamma[span] += (dz * xh).sum(0)
                d_beta[span] += dz.sum(0)
                dh = dz * gamma[span]
                d_x[i, on, span] = rstd * (dh - dh.mean() - xh * (dh * xh).mean())
    return {"y": y} if s["op"] == "norm" else {"y": y, "d_x": d_x, "d_gamma": d_gamma, "d_beta": d_beta}


def _exact_orth(g):
    """The polynomial applied to the singular values, one product of the steps' own factors at a time."""
    x = g.double()
    x = x / (torch.linalg.matrix_norm(x).view(-1, 1, 1) + _EPS_ORTH)
    tall = x.shape[1] > x.shape[2]
    a, b, c = _COEFFS
    eye = torch.eye(min(x.shape[1:]), dtype=torch.float64, device=x.device)
    for _ in range(_STEPS):
        xt = x.transpose(1, 2).contiguous()
        s = xt @ x if tall else x @ xt
        q = s @ (c * s + b * eye) + a * eye
        x = x @ q if tall else q @ x
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(s)
    if case["op"] == "orth":
        return {"out": [_exact_orth(g) for g in s["in"]]}
    weights, momenta = [], []
    for w, g, m in zip(s["weights"], s["grads"], s["momenta"]):
        m = _MU * m.double() + g.double()
        o = _exact_orth(g.double() + _MU * m if case["nesterov"] else m)
        weights.append((1 - _LR * _DECAY) * w.double() - _LR * max(1.0, w.shape[1] / w.shape[2]) ** 0.5 * o)
        momenta.append(m)
    return {"weights": weights, "momenta": momenta}
