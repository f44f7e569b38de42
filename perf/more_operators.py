"""Normalisation and weight update of a training step on verified weights: what is measured, and their plain forms.

Four operators: layer norm (with its root-mean-square form), its gradient with the sums over the rows, the AdamW step over a
ragged tensor set with states in 32 bits, and the same with states in 8 bits.  Widths and tensor lists are those of the
repository's synthetic weight files (24 layers of hidden size 2048, vocabulary 50257; hidden size 4096) and of its ragged
tensor set (sizes log-uniform from 4 KiB on).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 256                    # elements that share a scale of the 8-bit states; tensors' states start at multiples of it
TOP = 447.9995                 # what a block's largest value is scaled to: just below the largest code, 448
BETAS, EPS, DECAY, LR = (0.9, 0.999), 1e-8, 0.1, 1e-4

_context = None


def _ctx():
    """The program's verifier context: one per process, as a training program keeps it."""
    global _context
    if _context is None:
        from paper_2510_23938_b200 import binding
        _context = binding.Context(torch.cuda.current_device())
    return _context


# ------------------------------------------------------------------------------------------------------------------
# cases

def listed():
    return [
        # decoding one sequence: one token's hidden state, all latency
        {"name": "norm of 1 token", "op": "norm", "n": 1, "dim": 4096, "x": "bf16", "y": "bf16", "w": "bf16", "rms": True,
         "bias": False, "skew": 16},
        # one training step's tokens, the weight out of a weight file held as bytes, 8 bytes past a 16-byte boundary
        {"name": "norm of 8192 tokens", "op": "norm", "n": 8192, "dim": 2048, "x": "bf16", "y": "bf16", "w": "bf16",
         "rms": False, "bias": False, "skew": 8},
        # a long-context batch: the activations are 1 GB
        {"name": "norm of 131072 tokens", "op": "norm", "n": 131072, "dim": 4096, "x": "bf16", "y": "bf16", "w": "bf16",
         "rms": True, "bias": False, "skew": 16},
        # a short fine-tuning sequence
        {"name": "norm gradient of 509 tokens", "op": "grad", "n": 509, "dim": 2048, "x": "bf16", "y": "bf16", "w": "bf16",
         "rms": False, "bias": False, "add": False, "skew": 8},
        # a residual stream kept in 32 bits, an odd width, weight and bias
        {"name": "norm gradient of 6001 x 1023", "op": "grad", "n": 6001, "dim": 1023, "x": "f32", "y": "bf16", "w": "f32",
         "rms": False, "bias": True, "add": False, "skew": 4},
        # a pre-training step, the weight's gradient added to what earlier parts of the batch gave
        {"name": "norm gradient of 65536 tokens", "op": "grad", "n": 65536, "dim": 4096, "x": "bf16", "y": "bf16",
         "w": "bf16", "rms": True, "bias": False, "add": True, "skew": 16},
        # adapters of a small fine-tuning run: a few odd-sized tensors, latency counts
        {"name": "step of 7 small tensors", "op": "step", "set": "ragged", "n": 7, "low": 4 << 10, "high": 256 << 10,
         "w": "f32", "g": "f32", "bits": 32, "master": False, "skew": 0, "max_norm": 0.0, "stochastic": False},
        # 16-bit weights packed back to back at odd element offsets, 32-bit copies of them in the state
        {"name": "step of 200 packed tensors", "op": "step", "set": "ragged", "n": 200, "low": 4 << 10, "high": 4 << 20,
         "w": "bf16", "g": "bf16", "bits": 32, "master": True, "skew": 2, "max_norm": 1.0, "stochastic": False},
        # every tensor of the 24-layer file, updated in the file's bytes, clipped on the way
        {"name": "step of the 24-layer file", "op": "step", "set": "layers", "n": 24, "low": 0, "high": 0, "w": "bf16",
         "g": "bf16", "bits": 32, "master": False, "skew": 8, "max_norm": 1.0, "stochastic": False},
        # the small run with 8-bit states
        {"name": "8-bit step of 7 small tensors", "op": "step", "set": "ragged", "n": 7, "low": 4 << 10, "high": 256 << 10,
         "w": "bf16", "g": "bf16", "bits": 8, "master": False, "skew": 0, "max_norm": 0.0, "stochastic": True},
        # gradients accumulated in 32 bits, packed 16-bit weights rounded stochastically
        {"name": "8-bit step of 200 packed", "op": "step", "set": "ragged", "n": 200, "low": 4 << 10, "high": 4 << 20,
         "w": "bf16", "g": "f32", "bits": 8, "master": False, "skew": 2, "max_norm": 1.0, "stochastic": True},
        # the whole file with the smallest state there is: 10 bytes move per weight
        {"name": "8-bit step of 24-layer file", "op": "step", "set": "layers", "n": 24, "low": 0, "high": 0, "w": "bf16",
         "g": "bf16", "bits": 8, "master": False, "skew": 8, "max_norm": 1.0, "stochastic": True},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["norm", "grad", "step", "step"])
    if op == "step":
        w, g = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16")])
        bits = 32 if w == "f32" else rng.choice([8, 32])
        low = _log_uniform(rng, 64, 64 << 10)
        high = _log_uniform(rng, 4 * low, 16 << 20)
        most = max(1, min(1000, (1 << 30) // high))
        return {"op": op, "set": "ragged", "n": _log_uniform(rng, 1, most), "low": low, "high": high, "w": w, "g": g,
                "bits": bits, "master": bits == 32 and w != "f32" and rng.random() < 0.5, "skew": rng.choice([0, SIZE[w], 8]),
                "max_norm": rng.choice([0.0, 0.1, 1.0]), "stochastic": bits == 8 and rng.random() < 0.5}
    dim = rng.choice([2048, 4096, _log_uniform(rng, 32, 16384), 8 * _log_uniform(rng, 8, 1024)])
    n = min(_log_uniform(rng, 1, 131072), max(1, (1 << 28) // dim))
    x, y = rng.choice([("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f32")])
    case = {"op": op, "n": n, "dim": dim, "x": x, "y": y, "w": rng.choice([y, "f32"]), "rms": rng.random() < 0.5,
            "bias": rng.random() < 0.4, "skew": rng.choice([0, 4, 8, 16])}
    if op == "grad":
        case["add"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------------------------------------------------------
# inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, kind, g, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=kind, device="cuda").normal_(mean, std, generator=g)


def _prepare_norm(case, seed):
    g = _generator(seed)
    n, dim, kind, out = case["n"], case["dim"], TYPES[case["x"]], TYPES[case["y"]]
    weight = TYPES[case["w"]]
    skew = case["skew"] // SIZE[case["w"]]
    flat = _normal((skew + 2 * dim,), weight, g, 0.1, 1.0)
    s = {"case": case, "w": flat[skew:skew + dim], "b": flat[skew + dim:] if case["bias"] else None}
    s["x"] = _normal((n, dim), kind, g, 1.5, 0.3)
    # hidden states have a few columns of far larger values than the rest
    s["x"][:, ::97] *= 8
    if case["op"] == "norm":
        s["y"] = torch.empty(n, dim, dtype=out, device="cuda")
        s["mean"] = None if case["rms"] else torch.empty(n, dtype=torch.float32, device="cuda")
        s["rstd"] = torch.empty(n, dtype=torch.float32, device="cuda")
        return s
    s["dy"] = _normal((n, dim), out, g, 1e-3)
    step = max(1, (1 << 26) // dim)
    mean, rstd = [], []
    for x in s["x"].split(step):                        # what the forward pass left behind
        x = x.double()
        mu = torch.zeros_like(x[:, :1]) if case["rms"] else x.mean(1, keepdim=True)
        mean.append(mu[:, 0].float())
        rstd.append(((x - mu).square().mean(1) + 1e-5).rsqrt().float())
    s["mean"] = None if case["rms"] else torch.cat(mean)
    s["rstd"] = torch.cat(rstd)
    s["dx"] = torch.empty(n, dim, dtype=kind, device="cuda")
    for name in ("dw", "db"):
        s[name] = _normal((dim,), torch.float32, g, 1e-3) if case["add"] else torch.empty(dim, dtype=torch.float32, device="cuda")
    return s


def _set_elements(case):
    """Elements of each tensor of a set: a property of the model, the same for every seed."""
    if case["set"] == "layers":
        h, f, v = 2048, 8192, 50257
        layer = [h, h * h, h * h, h * h, h * h, h, f * h, h * f]
        return [v * h] + case["n"] * layer + [h]
    r = np.random.RandomState(case["n"] + case["high"] % 65521)
    nbytes = np.exp(r.uniform(math.log(case["low"]), math.log(case["high"]), case["n"]))
    return [max(1, int(b) // SIZE[case["w"]]) for b in nbytes]


def _prepare_step(case, seed):
    g = _generator(seed)
    kind, grad = TYPES[case["w"]], TYPES[case["g"]]
    counts = np.array(_set_elements(case), dtype=np.int64)
    starts = np.cumsum(counts) - counts                  # weights and gradients: tensors back to back
    room = (counts + BLOCK - 1) // BLOCK * BLOCK         # states: each tensor at a multiple of a block
    places = np.cumsum(room) - room
    total, size = int(counts.sum()), int(room.sum())
    skew = case["skew"] // SIZE[case["w"]]
    s = {"case": case, "size": size}
    s["w"] = _normal((skew + total,), kind, g, 0.02)[skew:]
    s["g"] = torch.empty(total, dtype=grad, device="cuda")
    m, root = torch.zeros(size, device="cuda"), torch.zeros(size, device="cuda")
    # the tensors of a model differ in gradient size by orders of magnitude
    spread = np.exp(np.random.RandomState((seed + 1) % (1 << 31)).uniform(math.log(1e-5), math.log(1e-2), len(counts)))
    for a, p, k, std in zip(starts.tolist(), places.tolist(), counts.tolist(), spread.tolist()):
        s["g"][a:a + k].normal_(0, std, generator=g)
        m[p:p + k].normal_(0, 0.3 * std, generator=g)
        root[p:p + k].log_normal_(math.log(std), 0.5, generator=g)
    if case["bits"] == 32:
        s["m"], s["v"] = m, root.square_()
        s["m_scales"] = s["v_scales"] = None
    else:
        for name, x in (("m", m), ("v", root)):
            rows = x.view(-1, BLOCK)
            scale = rows.abs().amax(1) / 448
            s[name] = (rows / scale.clamp_(min=1e-30).unsqueeze(1)).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scales"] = scale
    s["master"] = None
    if case["master"]:
        s["master"] = torch.zeros(size, device="cuda")
        for a, p, k in zip(starts.tolist(), places.tolist(), counts.tolist()):
            s["master"][p:p + k] = s["w"][a:a + k]
    as_bytes = lambda x, t: torch.from_numpy(x * SIZE[t]).cuda()  # noqa: E731
    s["offsets"], s["lengths"], s["grad_offsets"] = as_bytes(starts, case["w"]), as_bytes(counts, case["w"]), as_bytes(starts, case["g"])
    s["state_offsets"] = torch.from_numpy(places).cuda()
    s["starts"], s["counts"] = torch.from_numpy(starts).cuda(), torch.from_numpy(counts).cuda()
    s["step"] = torch.full((1,), 1000, dtype=torch.int64, device="cuda")
    s["seed"] = (seed * 0x9E3779B97F4A7C15 + 1) % (1 << 64)
    # the record of the gradients' norm (status, non-finite tensors, norm, scale, sum of squares, elements)
    s["norm"] = torch.zeros(32, dtype=torch.uint8, device="cuda")
    squares = torch.linalg.vector_norm(s["g"], dtype=torch.float64).square()
    s["norm"].view(torch.float32)[2], s["norm"].view(torch.float32)[3] = squares.sqrt().float(), 1.0
    s["norm"].view(torch.float64)[2], s["norm"].view(torch.int64)[3] = squares, total
    return s


def prepare(case, seed):
    return _prepare_step(case, seed) if case["op"] == "step" else _prepare_norm(case, seed)


# ------------------------------------------------------------------------------------------------------------------
# one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _norm_outputs(s):
    got = {"y": s["y"], "rstd": s["rstd"]}
    if s["mean"] is not None:
        got["mean"] = s["mean"]
    return got


def _grad_outputs(s):
    got = {"dx": s["dx"], "dw": s["dw"]}
    if s["b"] is not None:
        got["db"] = s["db"]
    return got


def _step_outputs(s):
    names = ("w", "m", "v", "m_scales", "v_scales", "master", "step")
    return {name: s[name] for name in names if s[name] is not None}


def _run_own(s):
    case, ctx = s["case"], _ctx()
    if case["op"] == "norm":
        ctx.layer_norm(s["x"], weight=s["w"], bias=s["b"], eps=1e-5, rms=case["rms"], out=s["y"], mean=s["mean"], rstd=s["rstd"])
        return _norm_outputs(s)
    if case["op"] == "grad":
        ctx.layer_norm_grad(s["dy"], s["x"], s["mean"], s["rstd"], weight=s["w"], rms=case["rms"], out=s["dx"],
                            weight_grad=s["dw"], bias_grad=s["db"] if case["bias"] else None, accumulate=case["add"])
        return _grad_outputs(s)
    ctx.adamw_step(s["w"], s["offsets"], s["lengths"], s["g"], s["grad_offsets"], state_offsets=s["state_offsets"], m=s["m"],
                   v=s["v"], step=s["step"], m_scales=s["m_scales"], v_scales=s["v_scales"], master=s["master"], lr=LR,
                   betas=BETAS, eps=EPS, weight_decay=DECAY, norm=s["norm"] if case["max_norm"] else None,
                   max_norm=case["max_norm"] or None, stochastic=case["stochastic"], seed=s["seed"])
    return _step_outputs(s)


def _run_plain(s):
    op = s["case"]["op"]
    return _plain_norm(s) if op == "norm" else _plain_grad(s) if op == "grad" else _plain_step(s)


def _plain_norm(s):
    case = s["case"]
    x = s["x"].float()
    if not case["rms"]:
        mean = x.mean(1)
        s["mean"].copy_(mean)
        x = x - mean.unsqueeze(1)
    rstd = (x.square().mean(1) + 1e-5).rsqrt()
    s["rstd"].copy_(rstd)
    y = x * rstd.unsqueeze(1) * s["w"].float()
    s["y"].copy_(y if s["b"] is None else y + s["b"].float())
    return _norm_outputs(s)


def _plain_grad(s):
    case = s["case"]
    x, dy = s["x"].float(), s["dy"].float()
    rstd = s["rstd"].unsqueeze(1)
    h = x * rstd if case["rms"] else (x - s["mean"].unsqueeze(1)) * rstd
    dw = (dy * h).sum(0)
    s["dw"].copy_(dw + s["dw"] if case["add"] else dw)
    if case["bias"]:
        db = dy.sum(0)
        s["db"].copy_(db + s["db"] if case["add"] else db)
    p = dy * s["w"].float()
    dx = p - h * (p * h).mean(1, keepdim=True)
    if not case["rms"]:
        dx = dx - p.mean(1, keepdim=True)
    s["dx"].copy_(dx * rstd)
    return _grad_outputs(s)


# The random numbers of a step: 32-bit words from a hash of (seed, number of the step, element).  Elements are taken in
# groups of eight; word k of group q is b + (k + 1) a with b = mix(q ^ K0), a = mix(b + K1); words 0 to 7 round the first
# moments of the group's elements, 8 to 15 the roots of the second, 16 to 23 the weights.

GOLDEN = 0x9E3779B9


def _signed(x):
    x &= 0xffffffff
    return x - (1 << 32) if x >> 31 else x


def _mix(x):
    """A hash of 32-bit words (int32, wrapping)."""
    x = x ^ ((x >> 16) & 0xffff)
    x = x * _signed(0x6A09E667)
    x = x ^ ((x >> 15) & 0x1ffff)
    x = x * _signed(0xBB67AE85)
    return x ^ ((x >> 16) & 0xffff)


def _words(s, first):
    """Words first .. first + 7 of every group: one per element (int32)."""
    number = s["step"] + 1
    low = number.to(torch.int32)
    seed = torch.full_like(low, _signed(s["seed"]))
    k0 = _mix(_mix(_mix(seed + _signed(GOLDEN)) + _signed(s["seed"] >> 32)) + low)
    k1 = _mix(k0 + (number >> 32).to(torch.int32) + _signed(GOLDEN))
    b = _mix(torch.arange(s["size"] // 8, dtype=torch.int32, device="cuda") ^ k0)
    a = _mix(b + k1)
    k = torch.arange(first + 1, first + 9, dtype=torch.int32, device="cuda")
    return (b.unsqueeze(1) + a.unsqueeze(1) * k).view(-1)


def _plain_codes(x, words, s, name):
    """x in blocks as e4m3 codes (stored to s[name]) and scales: the 20 bits behind a code's last are rounded by 20 random
    ones; a moment that is not zero keeps a code that is not zero where `name` is the root of v."""
    rows = x.view(-1, BLOCK)
    top = rows.abs().amax(1)
    safe = top.clamp(min=2.0 ** -110)
    scaled = rows.abs() * (TOP / safe).unsqueeze(1) * 2.0 ** -120             # codes are the upper bits of such a float
    code = (scaled.view(torch.int32).view(-1) + ((words >> 12) & 0xfffff)) >> 20
    if name == "v":
        code = torch.maximum(code, (x > 0).to(torch.int32))
    code = torch.where(x < 0, code | 128, code).to(torch.uint8)
    s[name].view(torch.uint8).copy_(code)
    s[name + "_scales"].copy_(torch.where(top > 0, safe * (1.0 / TOP), torch.zeros_like(top)))


def _plain_weights(x, words, kind):
    """x rounded to a 16-bit type by random bits in the place of those that go."""
    if kind is torch.bfloat16:
        return ((x.view(torch.int32) + ((words >> 16) & 0xffff)) & -65536).view(torch.float32).to(kind)
    code = ((x.abs() * 2.0 ** -112).view(torch.int32) + ((words >> 19) & 0x1fff)) >> 13
    return torch.where(x < 0, code | -32768, code).to(torch.int16).view(kind)


def _plain_step(s):
    case, size = s["case"], s["size"]
    packed = size != s["w"].numel()
    if packed:                                           # the elements' places in the state
        tensor = torch.repeat_interleave(torch.arange(s["counts"].numel(), device="cuda"), s["counts"], output_size=s["w"].numel())
        place = torch.arange(s["w"].numel(), device="cuda") + (s["state_offsets"] - s["starts"])[tensor]
    spread = lambda x: torch.zeros(size, device="cuda").index_copy_(0, place, x) if packed else x  # noqa: E731
    gather = lambda x: x[place] if packed else x  # noqa: E731
    number = (s["step"] + 1).double()
    g = spread(s["g"].float())
    if case["max_norm"]:
        norm = s["norm"].view(torch.float64)[2].sqrt()
        g = g * torch.where(norm <= case["max_norm"], torch.ones_like(norm), case["max_norm"] / norm).float()
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scales"].unsqueeze(1)).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scales"].unsqueeze(1)).view(-1).square_()
    m = m * BETAS[0] + g * (1 - BETAS[0])
    v = v * BETAS[1] + g * g * (1 - BETAS[1])
    root = v.sqrt()
    size_of_step = (LR / (1 - BETAS[0] ** number)).float()
    update = m * size_of_step / (root * (1 - BETAS[1] ** number).rsqrt().float() + EPS)
    w = s["master"] if case["master"] else spread(s["w"].float())
    w = w * (1 - LR * DECAY) - update
    if case["master"]:
        s["master"].copy_(w)
    s["w"].copy_(gather(_plain_weights(w, _words(s, 16), TYPES[case["w"]]) if case["stochastic"] else w))
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        _plain_codes(m, _words(s, 0), s, "m")
        _plain_codes(root, _words(s, 8), s, "v")
    s["step"].add_(1)
    return _step_outputs(s)


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    if case["op"] == "step":
        counts = _set_elements(case)
        elements = sum(counts)
        w, g = SIZE[case["w"]], SIZE[case["g"]]
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        weights = w + 8 if case["master"] else 2 * w
        return {"bytes": elements * (weights + g + state) + 32 * len(counts), "flops": elements * 14}
    n, dim = case["n"], case["dim"]
    x, y = SIZE[case["x"]], SIZE[case["y"]]
    vectors = dim * SIZE[case["w"]] * (2 if case["bias"] else 1)
    stats = n * (4 if case["rms"] else 8)
    if case["op"] == "norm":
        return {"bytes": n * dim * (x + y) + vectors + stats, "flops": n * dim * 7}
    sums = dim * 4 * (2 if case["bias"] else 1) * (2 if case["add"] else 1)
    return {"bytes": n * dim * (2 * x + y) + dim * SIZE[case["w"]] + stats + sums, "flops": n * dim * 13}


# ------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_step(s) if case["op"] == "step" else _exact_norm(s)


def _exact_norm(s):
    case = s["case"]
    w = s["w"].double()
    part = max(1, (1 << 27) // case["dim"])
    rows = range(0, case["n"], part)
    if case["op"] == "norm":
        y, mean, rstd = torch.empty(case["n"], case["dim"], dtype=torch.float64, device="cuda"), [], []
        for a in rows:
            x = s["x"][a:a + part].double()
            mu = torch.zeros(x.shape[0], 1, dtype=torch.float64, device="cuda") if case["rms"] else x.mean(1, keepdim=True)
            r = 1 / ((x - mu).pow(2).mean(1, keepdim=True) + 1e-5).sqrt()
            y[a:a + part] = (x - mu) * r * w
            mean.append(mu[:, 0])
            rstd.append(r[:, 0])
        if s["b"] is not None:
            y += s["b"].double()
        got = {"y": y, "rstd": torch.cat(rstd)}
        return got if case["rms"] else {**got, "mean": torch.cat(mean)}
    dx = torch.empty(case["n"], case["dim"], dtype=torch.float64, device="cuda")
    dw, db = (s[k].double() if case["add"] else torch.zeros(case["dim"], dtype=torch.float64, device="cuda") for k in ("dw", "db"))
    for a in rows:
        x, dy, r = s["x"][a:a + part].double(), s["dy"][a:a + part].double(), s["rstd"][a:a + part].double()[:, None]
        h = (x if case["rms"] else x - s["mean"][a:a + part].double()[:, None]) * r
        p = dy * w
        inner = p - h * (p * h).mean(1, keepdim=True)
        dx[a:a + part] = r * (inner if case["rms"] else inner - p.mean(1, keepdim=True))
        dw += torch.einsum("ij,ij->j", dy, h)
        db += dy.sum(0)
    return {"dx": dx, "dw": dw, "db": db} if case["bias"] else {"dx": dx, "dw": dw}


def _hash64(x):
    """The hash on 32-bit words held in int64."""
    low = 0xffffffff
    x = x ^ (x >> 16)
    x = x * 0x6A09E667 & low
    x = x ^ (x >> 15)
    x = x * 0xBB67AE85 & low                             # the wrapped 64-bit product has the right lower half
    return x ^ (x >> 16)


def _words64(s, first, a, b):
    """The words of the state elements a .. b - 1 as int64."""
    low, number, seed = 0xffffffff, int(s["step"][0]) + 1, s["seed"]
    one = lambda x: int(_hash64(torch.tensor(x & low)))  # noqa: E731
    k0 = one(one(one(seed + GOLDEN) + (seed >> 32)) + number)
    k1 = one(k0 + (number >> 32) + GOLDEN)
    group = torch.arange(a // 8, b // 8, device="cuda")
    base = _hash64(group ^ k0)
    stride = _hash64((base + k1) & low)
    k = torch.arange(first + 1, first + 9, device="cuda")
    return ((base[:, None] + stride[:, None] * k) & low).view(-1)


def _on_grid(x, digits, lowest, random):
    """|x| on the grid of floats with `digits` binary places behind the first and exponents from `lowest` on, rounded up with
    the probability `random` (in [0, 1)) exceeds what is missing."""
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** (lowest - 1)))).clamp(min=lowest)
    unit = torch.exp2(e - digits)
    return torch.floor(x / unit + random) * unit


def _exact_codes(x, words, root):
    rows = x.view(-1, BLOCK)
    top = rows.abs().amax(1, keepdim=True)
    safe = top.clamp(min=2.0 ** -110)
    code = _on_grid(rows.abs() * (TOP / safe), 3, -6, ((words >> 12).double() / 2 ** 20).view(-1, BLOCK))
    if root:
        code = torch.where(rows > 0, code.clamp(min=2.0 ** -9), code)
    return (code * rows.sign()).view(-1), torch.where(top > 0, safe / TOP, torch.zeros_like(top))[:, 0]


def _exact_step(s):
    case, size = s["case"], s["size"]
    number = int(s["step"][0]) + 1
    factor = 1.0
    if case["max_norm"]:
        norm = math.sqrt(float(s["norm"].view(torch.float64)[2]))
        factor = 1.0 if norm <= case["max_norm"] else case["max_norm"] / norm
    starts, counts, places = (s[k].tolist() for k in ("starts", "counts", "state_offsets"))
    part = 1 << 26
    got = {k: [] for k in ("m", "v", "m_scales", "v_scales", "master")}
    out = torch.empty(s["w"].numel(), dtype=torch.float64, device="cuda")
    for a in range(0, size, part):                       # state elements a .. b - 1
        b = min(size, a + part)
        here = [(max(p, a), min(p + k, b), t) for p, k, t in zip(places, counts, starts) if p < b and p + k > a]
        at = [(i - a, j - a, i - p + t, j - p + t) for (i, j, t), p in
              zip(here, [p for p, k in zip(places, counts) if p < b and p + k > a])]
        g, w = torch.zeros(b - a, dtype=torch.float64, device="cuda"), torch.zeros(b - a, dtype=torch.float64, device="cuda")
        for i, j, x, y in at:
            g[i:j], w[i:j] = s["g"][x:y].double() * factor, s["w"][x:y].double()
        if case["master"]:
            w = s["master"][a:b].double()
        m, v = s["m"][a:b].double(), s["v"][a:b].double()
        if case["bits"] == 8:
            m = (m.view(-1, BLOCK) * s["m_scales"][a // BLOCK:b // BLOCK].double()[:, None]).view(-1)
            v = (v.view(-1, BLOCK) * s["v_scales"][a // BLOCK:b // BLOCK].double()[:, None]).view(-1).pow(2)
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g.pow(2)
        right = (v / (1 - BETAS[1] ** number)).sqrt() + EPS
        w = w - LR * DECAY * w - LR * (m / (1 - BETAS[0] ** number)) / right
        got["master"].append(w)
        if case["stochastic"]:
            words = _words64(s, 16, a, b)
            if case["w"] == "bf16":
                w = _on_grid(w.abs(), 7, -126, (words >> 16).double() / 2 ** 16) * w.sign()
            else:
                w = _on_grid(w.abs(), 10, -14, (words >> 19).double() / 2 ** 13) * w.sign()
        for i, j, x, y in at:
            out[x:y] = w[i:j]
        if case["bits"] == 8:
            m, m_scales = _exact_codes(m, _words64(s, 0, a, b), False)
            v, v_scales = _exact_codes(v.sqrt(), _words64(s, 8, a, b), True)
            got["m_scales"].append(m_scales)
            got["v_scales"].append(v_scales)
        got["m"].append(m)
        got["v"].append(v)
    answer = {"w": out, "step": s["step"] + 1, **{k: torch.cat(x) for k, x in got.items() if x and k != "master"}}
    if case["master"]:
        answer["master"] = torch.cat(got["master"])
    return answer
