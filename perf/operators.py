"""The operators of a training step on verified weights: what is measured, and their plain forms.

Four operators: the embedding lookup with scaling, its gradient by sorted tokens (dense or as the touched rows only),
the global gradient norm over a ragged tensor set, and clipping by it.  Table shapes and tensor lists are those of the
repository's synthetic weight files (24 layers of hidden size 2048, vocabulary 50257; hidden size 4096, vocabulary
128256) and of its ragged tensor set (sizes log-uniform from 4 KiB to 64 MiB).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
ROW = 2048          # elements of one row of the plain form's view of a gradient buffer

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
        # decoding one sequence: one token's row, no arithmetic to speak of, all latency
        {"name": "lookup 1 token", "op": "lookup", "n": 1, "rows": 128256, "dim": 4096, "type": "bf16", "out": "bf16",
         "scale": 1.0, "index": "i64", "skew": 16},
        # a small decoding batch out of a weight file held as bytes: the table starts 8 bytes past a 16-byte boundary
        {"name": "lookup 61 tokens in a file", "op": "lookup", "n": 61, "rows": 50257, "dim": 2048, "type": "bf16",
         "out": "f32", "scale": 1.0, "index": "i32", "skew": 8},
        # one training step's tokens, activations scaled by the square root of the hidden size
        {"name": "lookup 8192 tokens", "op": "lookup", "n": 8192, "rows": 128256, "dim": 4096, "type": "bf16",
         "out": "bf16", "scale": 64.0, "index": "i64", "skew": 8},
        # a long-context batch: the activations alone are 1 GB
        {"name": "lookup 131072 tokens", "op": "lookup", "n": 131072, "rows": 128256, "dim": 4096, "type": "bf16",
         "out": "bf16", "scale": 64.0, "index": "i64", "skew": 16},
        # a short fine-tuning sequence: the touched rows of the smaller table
        {"name": "gradient rows of 509 tokens", "op": "rows", "n": 509, "rows": 50257, "dim": 2048, "type": "bf16",
         "out": "bf16", "scale": 1.0, "index": "i64", "pad": 0.0},
        # a tied head: the lookup's share is added to a 32-bit gradient that is there already
        {"name": "gradient of 8192 tokens added", "op": "dense", "n": 8192, "rows": 50257, "dim": 2048, "type": "bf16",
         "out": "f32", "scale": 1.0, "index": "i64", "pad": 0.0, "add": True},
        # a padded fine-tuning batch: a quarter of the tokens are padding and give no gradient
        {"name": "gradient rows of 16384 tokens", "op": "rows", "n": 16384, "rows": 128256, "dim": 4096, "type": "bf16",
         "out": "bf16", "scale": 64.0, "index": "i64", "pad": 0.25},
        # a pre-training step: the whole table's gradient, untouched rows zero
        {"name": "gradient of 65536 tokens", "op": "dense", "n": 65536, "rows": 128256, "dim": 4096, "type": "bf16",
         "out": "bf16", "scale": 64.0, "index": "i64", "pad": 0.0, "add": False},
        # adapters of a small fine-tuning run: a few odd-sized tensors, latency counts
        {"name": "clip of 7 small tensors", "op": "clip", "set": "ragged", "n": 7, "low": 4 << 10, "high": 256 << 10,
         "type": "f32", "out": "f32", "packed": True, "max_norm": 0.1},
        # the norm of one step's gradients of the 24-layer file, 194 tensors, for logging and the skip decision
        {"name": "norm of the 24-layer file", "op": "norm", "set": "layers", "n": 24, "low": 0, "high": 0, "type": "bf16",
         "out": "bf16", "packed": False, "max_norm": 1.0},
        # gradients packed back to back at odd element offsets, clipped in their own type
        {"name": "clip of 200 packed tensors", "op": "clip", "set": "ragged", "n": 200, "low": 4 << 10, "high": 4 << 20,
         "type": "bf16", "out": "bf16", "packed": True, "max_norm": 1.0},
        # a ragged set accumulated in 32 bits, clipped and handed on in 16 bits
        {"name": "clip of 1000 ragged tensors", "op": "clip", "set": "ragged", "n": 1000, "low": 4 << 10, "high": 64 << 20,
         "type": "f32", "out": "bf16", "packed": False, "max_norm": 1.0},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["lookup", "rows", "dense", "norm", "clip"])
    kind, out = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
    if op in ("norm", "clip"):
        kind, out = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f16", "f16"), ("f32", "f32")])
        low = _log_uniform(rng, 64, 64 << 10)
        high = _log_uniform(rng, 4 * low, 16 << 20)
        most = max(1, min(1000, (2 << 30) // high))
        return {"op": op, "set": "ragged", "n": _log_uniform(rng, 1, most), "low": low, "high": high, "type": kind,
                "out": out if op == "clip" else kind, "packed": rng.random() < 0.4,
                "max_norm": rng.choice([0.1, 1.0, 1e9])}
    dim = rng.choice([2048, 4096, _log_uniform(rng, 1, 8192), 8 * _log_uniform(rng, 8, 1024)])
    rows = rng.choice([50257, 128256, _log_uniform(rng, 2, 100000)])
    rows = max(2, min(rows, (1 << 30) // (4 * dim)))
    n = min(_log_uniform(rng, 1, 131072), max(1, (1 << 30) // (4 * dim)))
    case = {"op": op, "n": n, "rows": rows, "dim": dim, "type": kind, "out": out,
            "scale": rng.choice([1.0, math.sqrt(dim)]), "index": rng.choice(["i32", "i64"])}
    if op == "lookup":
        case["skew"] = rng.choice([0, SIZE[kind], 8, 16])
    else:
        case["pad"] = rng.choice([0.0, 0.3, 0.9])
    if op == "dense":
        case["add"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------------------------------------------------------
# inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _tokens(case, g):
    """Token frequencies fall with the token's number as in text: P(r) proportional to log((r + 2) / (r + 1))."""
    u = torch.rand(case["n"], generator=g, device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(case["rows"] + 1)).floor() - 1).clamp_(0, case["rows"] - 1).to(torch.int64)
    if case.get("pad"):
        t[torch.rand(case["n"], generator=g, device="cuda") < case["pad"]] = case["rows"] - 1
    return t.to(torch.int32 if case["index"] == "i32" else torch.int64)


def _set_lengths(case):
    """Elements of each tensor of a gradient set: a property of the model, the same for every seed."""
    if case["set"] == "layers":
        h, f, v = 2048, 8192, 50257
        layer = [h, h * h, h * h, h * h, h * h, h, f * h, h * f]
        return [v * h] + case["n"] * layer + [h]
    r = np.random.RandomState(case["n"] + case["high"] % 65521)
    nbytes = np.exp(r.uniform(math.log(case["low"]), math.log(case["high"]), case["n"]))
    return [max(1, int(b) // SIZE[case["type"]]) for b in nbytes]


def _set_starts(case, lengths):
    """First element of each tensor in the flat buffer, and the buffer's length: back to back, or each tensor at a
    multiple of ROW elements with zeros behind it."""
    room = np.array(lengths, dtype=np.int64)
    if not case["packed"]:
        room = (room + ROW - 1) // ROW * ROW
    ends = np.cumsum(room)
    return (ends - room).tolist(), int(ends[-1])


def prepare(case, seed):
    g = _generator(seed)
    kind, out = TYPES[case["type"]], TYPES[case["out"]]
    s = {"case": case}
    if case["op"] in ("lookup", "rows", "dense"):
        n, rows, dim = case["n"], case["rows"], case["dim"]
        s["tokens"] = _tokens(case, g)
        if case["op"] == "lookup":
            skew = case["skew"] // SIZE[case["type"]]
            flat = torch.empty(skew + rows * dim, dtype=kind, device="cuda").normal_(0, 0.02, generator=g)
            s["table"] = flat[skew:].view(rows, dim)
            s["out"] = torch.empty(n, dim, dtype=out, device="cuda")
            return s
        s["grad"] = torch.empty(n, dim, dtype=kind, device="cuda").normal_(0, 1e-3, generator=g)
        s["padding"] = rows - 1 if case["pad"] else None
        if case["op"] == "rows":
            cap = min(n, rows)
            s["rows"] = torch.empty(cap, dtype=torch.int64, device="cuda")
            s["count"] = torch.empty(1, dtype=torch.int64, device="cuda")
            s["out"] = torch.empty(cap, dim, dtype=out, device="cuda")
        else:
            s["out"] = torch.empty(rows, dim, dtype=out, device="cuda")
            if case["add"]:
                s["out"].normal_(0, 1e-3, generator=g)
        return s
    lengths = _set_lengths(case)
    starts, total = _set_starts(case, lengths)
    s["host_lengths"], s["host_starts"] = lengths, starts
    s["starts"] = torch.tensor(starts, dtype=torch.int64, device="cuda")
    s["counts"] = torch.tensor(lengths, dtype=torch.int64, device="cuda")
    s["flat"] = torch.zeros(total, dtype=kind, device="cuda")
    # the tensors of a model differ in gradient size by orders of magnitude
    spread = np.exp(np.random.RandomState((seed + 1) % (1 << 31)).uniform(math.log(1e-5), math.log(1e-2), len(lengths)))
    for a, m, std in zip(starts, lengths, spread):
        s["flat"][a:a + m].normal_(0, float(std), generator=g)
    s["offsets"] = s["starts"] * SIZE[case["type"]]      # bytes, as the per-tensor digests take them
    s["lengths"] = s["counts"] * SIZE[case["type"]]
    s["norms"] = torch.empty(len(lengths), dtype=torch.float32, device="cuda")
    s["result"] = torch.zeros(32, dtype=torch.uint8, device="cuda")
    if case["op"] == "clip":
        s["out"] = torch.zeros(total, dtype=out, device="cuda")
        s["out_offsets"] = s["starts"] * SIZE[case["out"]]
    return s


# ------------------------------------------------------------------------------------------------------------------
# one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, ctx = s["case"], _ctx()
    if case["op"] == "lookup":
        return ctx.embedding(s["table"], s["tokens"], scale=case["scale"], out=s["out"])
    if case["op"] == "rows":
        rows, grad, count = ctx.embedding_grad_rows(s["grad"], s["tokens"], case["rows"], scale=case["scale"],
                                                    padding_row=s["padding"], rows=s["rows"], out=s["out"],
                                                    count=s["count"])
        return {"rows": rows, "grad": grad, "count": count}
    if case["op"] == "dense":
        return ctx.embedding_grad(s["grad"], s["tokens"], case["rows"], scale=case["scale"], padding_row=s["padding"],
                                  out=s["out"], accumulate=case["add"])
    if case["op"] == "norm":
        ctx.grad_norm(s["flat"], s["offsets"], s["lengths"], s["result"], norms=s["norms"])
    else:
        ctx.grad_clip(s["flat"], s["offsets"], s["lengths"], case["max_norm"], s["result"], norms=s["norms"],
                      out=s["out"], out_offsets=s["out_offsets"])
    words = s["result"].view(torch.int32)
    got = {"norm": s["result"].view(torch.float32)[2:4], "nonfinite": words[1:2], "norms": s["norms"]}
    if case["op"] == "clip":
        got["grads"] = s["out"]
    return got


def _run_plain(s):
    case = s["case"]
    if case["op"] == "lookup":
        s["out"].copy_(s["table"][s["tokens"]].float() * case["scale"])
        return s["out"]
    if case["op"] == "rows":
        return _plain_rows(s)
    if case["op"] == "dense":
        return _plain_dense(s)
    return _plain_set(s)


def _plain_live(s):
    """The tokens' gradients in 32 bits, zero where the token is padding."""
    g = s["grad"].float()
    if s["padding"] is not None:
        g = g * (s["tokens"] != s["padding"]).unsqueeze(1)
    return g


def _plain_dense(s):
    case = s["case"]
    total = torch.zeros(case["rows"], case["dim"], dtype=torch.float32, device="cuda")
    total.index_add_(0, s["tokens"].long(), _plain_live(s))
    total *= case["scale"]
    if case["add"]:
        total += s["out"]
    s["out"].copy_(total)
    return s["out"]


def _plain_rows(s):
    case, n = s["case"], s["case"]["n"]
    cap = s["rows"].numel()
    tokens, order = torch.sort(s["tokens"].long(), stable=True)
    live = tokens != (-1 if s["padding"] is None else s["padding"])      # padding is the last row: it sorts behind the rest
    head = torch.ones(n, dtype=torch.bool, device="cuda")
    head[1:] = tokens[1:] != tokens[:-1]
    place = torch.cumsum(head, 0) - 1
    head &= live
    total = torch.zeros(n, case["dim"], dtype=torch.float32, device="cuda")
    total.index_add_(0, place, _plain_live(s)[order])
    total *= case["scale"]
    spare = torch.full((n + 1,), -1, dtype=torch.int64, device="cuda")
    spare.scatter_(0, torch.where(head, place, n), tokens)               # the last place takes what is no head
    s["rows"].copy_(spare[:cap])
    s["count"].copy_(head.sum())
    s["out"].copy_(total[:cap])
    return {"rows": s["rows"], "grad": s["out"], "count": s["count"]}


def _plain_squares(s):
    """Sum of squares of each tensor, in 32 bits, through rows of ROW elements."""
    case, flat = s["case"], s["flat"]
    per = (s["counts"] + ROW - 1) // ROW                                  # rows of each tensor
    total = sum(-(-m // ROW) for m in s["host_lengths"])
    tensor = torch.repeat_interleave(torch.arange(per.numel(), device="cuda"), per, output_size=total)
    if case["packed"]:
        first = torch.cumsum(per, 0) - per
        at = (torch.arange(total, device="cuda") - first[tensor]) * ROW   # the row's place within its tensor
        column = at.unsqueeze(1) + torch.arange(ROW, device="cuda")
        inside = column < s["counts"][tensor].unsqueeze(1)
        rows = flat[(s["starts"][tensor].unsqueeze(1) + column).clamp_(max=flat.numel() - 1)].float() * inside
    else:
        rows = flat.view(total, ROW).float()                              # tensors start at rows; zeros fill their last one
    return torch.zeros(per.numel(), dtype=torch.float32, device="cuda").index_add_(0, tensor, rows.square().sum(1))


def _plain_set(s):
    case = s["case"]
    squares = _plain_squares(s)
    norm = squares.sum().sqrt()
    scale = torch.where(norm <= case["max_norm"], torch.ones_like(norm), case["max_norm"] / norm)
    got = {"norm": torch.stack([norm, scale if case["op"] == "clip" else torch.ones_like(norm)]),
           "nonfinite": (~torch.isfinite(squares)).sum().to(torch.int32).reshape(1), "norms": squares.sqrt()}
    if case["op"] == "clip":
        s["out"].copy_(s["flat"].float() * scale)
        got["grads"] = s["out"]
    return got


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def _distinct(case):
    """Expected number of distinct tokens, padding not among them."""
    n = case["n"] * (1.0 - case.get("pad", 0.0))
    r = np.arange(case["rows"], dtype=np.float64)
    p = np.log((r + 2) / (r + 1)) / math.log(case["rows"] + 1)
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    if case["op"] in ("norm", "clip"):
        elements = sum(_set_lengths(case))
        nbytes = elements * (SIZE[case["type"]] + (SIZE[case["out"]] if case["op"] == "clip" else 0))
        return {"bytes": nbytes + 24 * case["n"], "flops": elements * (3 if case["op"] == "clip" else 2)}
    n, dim = case["n"], case["dim"]
    inner, outer, index = SIZE[case["type"]], SIZE[case["out"]], 4 if case["index"] == "i32" else 8
    distinct = _distinct(case)
    if case["op"] == "lookup":
        return {"bytes": n * index + dim * (distinct * inner + n * outer), "flops": n * dim}
    live = n * (1.0 - case["pad"])
    if case["op"] == "rows":
        written = min(n, case["rows"]) * (dim * outer + 8)
    else:
        written = dim * outer * (2 * distinct if case["add"] else case["rows"])
    return {"bytes": n * index + live * dim * inner + written, "flops": live * dim + distinct * dim}


# ------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "lookup":
        return torch.nn.functional.embedding(s["tokens"].long(), s["table"].double()) * case["scale"]
    if case["op"] in ("rows", "dense"):
        tokens, grad = s["tokens"].long(), s["grad"].double() * case["scale"]
        if s["padding"] is not None:
            keep = tokens != s["padding"]
            tokens, grad = tokens[keep], grad[keep]
        if case["op"] == "dense":
            total = s["out"].double() if case["add"] else torch.zeros(case["rows"], case["dim"], dtype=torch.float64,
                                                                      device="cuda")
            return total.index_put_((tokens,), grad, accumulate=True)
        distinct, place = torch.unique(tokens, sorted=True, return_inverse=True)
        cap = min(case["n"], case["rows"])
        rows = torch.full((cap,), -1, dtype=torch.int64, device="cuda")
        rows[:distinct.numel()] = distinct
        total = torch.zeros(cap, case["dim"], dtype=torch.float64, device="cuda").index_put_((place,), grad, accumulate=True)
        return {"rows": rows, "grad": total, "count": torch.tensor([distinct.numel()], device="cuda")}
    norms = torch.stack([torch.linalg.vector_norm(s["flat"][a:a + m], dtype=torch.float64)
                         for a, m in zip(s["host_starts"], s["host_lengths"])])
    norm = torch.linalg.vector_norm(norms)
    bad = (~torch.isfinite(norms)).sum().to(torch.int32).reshape(1)
    limit = float(case["max_norm"])
    scale = torch.ones_like(norm) if case["op"] == "norm" or float(norm) <= limit else limit / norm
    got = {"norm": torch.stack([norm, scale]), "nonfinite": bad, "norms": norms}
    if case["op"] == "clip":
        got["grads"] = s["flat"].double() * scale
    return got
