"""Fine-tuning steps on verified weights: verify, look up, differentiate, clip, update, re-verify what changed.

    python examples/verified_finetune_step.py [--layers gpt] [--steps 3] [--norm] [--optimizer adamw8]

The weights are one byte blob in device memory (a weight file: header, tensor index, bf16 tensors back to back) that has
been verified against its manifest; every tensor used below is a view into those bytes.  A step trains two of them,
the embedding table and one projection, on a regression target:

    hidden = sqrt(h) * table[tokens]        ctx.embedding
    y      = hidden @ up^T                  (library product; with --norm a root-mean-square norm of hidden before it,
                                            ctx.layer_norm and ctx.layer_norm_grad, whose weight is trained too)
    rows, d_table = gradient of the lookup  ctx.embedding_grad_rows: the touched rows only
    norm over both gradients, clipping      ctx.grad_clip
    table[rows] -= lr * d_table, up -= ...  in place, in the verified bytes
    the chunks those bytes lie in           ctx.tree_update -> new root

With --optimizer adamw (moments in 32 bits) or adamw8 (in 8) the last three of these are the norm of all gradients
(ctx.grad_norm) and one ctx.adamw_step over the trained tensors, in place in the verified bytes, which clips on the way; the
table's gradient is then the whole table's (ctx.embedding_grad) and every chunk of a trained tensor is dirty.

Everything is a function of the inputs bit for bit, so replicas that make the same steps hold the same root.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2510_23938_b200 import binding, inputs  # noqa: E402


def tensor_view(blob: torch.Tensor, table, name: str, shapes) -> torch.Tensor:
    """A bf16 tensor of the weight file as a view into its bytes."""
    offset, nbytes = next((o, n) for key, o, n in table if key == name)
    return blob[offset:offset + nbytes].view(torch.bfloat16).view(shapes[name])


def chunks_of(starts: torch.Tensor, nbytes: int, chunk_bytes: int) -> torch.Tensor:
    """Indices of the chunks that hold any of the `nbytes` bytes from each start."""
    first, last = starts // chunk_bytes, (starts + nbytes - 1) // chunk_bytes
    longest = (nbytes - 1) // chunk_bytes + 2
    every = first[:, None] + torch.arange(longest, device=starts.device)
    return torch.unique(every[every <= last[:, None]])


def forward(ctx: binding.Context, weights, up, norm, tokens, target) -> dict:
    """The loss and what its gradients need."""
    hidden = ctx.embedding(weights, tokens, scale=math.sqrt(weights.shape[1]))
    s = {"hidden": hidden, "inner": hidden, "rstd": None}
    if norm is not None:
        s["rstd"] = torch.empty(tokens.numel(), device=hidden.device)
        s["inner"] = ctx.layer_norm(hidden, weight=norm, rms=True, rstd=s["rstd"])
    s["error"] = (s["inner"] @ up.t()).float() - target
    s["loss"] = s["error"].square().mean()
    return s


def backward(ctx: binding.Context, s: dict, up, norm) -> tuple:
    """Gradients of the projection, of the lookup's result and of the norm's weight (None without one)."""
    d_y = (s["error"] * (2.0 / s["error"].numel())).to(torch.bfloat16)
    d_up, d_hidden, d_norm = d_y.t() @ s["inner"], d_y @ up, None
    if norm is not None:
        d_norm = torch.empty_like(norm)
        d_hidden = ctx.layer_norm_grad(d_hidden, s["hidden"], None, s["rstd"], weight=norm, rms=True, weight_grad=d_norm)
    return d_up, d_hidden, d_norm


def run(ctx: binding.Context, tensors, embedding: str, projection: str, chunk_bytes: int, steps: int, n_tokens: int,
        lr: float = 2.0, max_norm: float = 0.02, seed: int = 1, norm_weight: str | None = None, optimizer: str = "sgd") -> dict:
    device = f"cuda:{ctx.device}"
    shapes = dict(tensors)
    blob, table = inputs.weight_file(tensors, seed, device)
    offset_of = {name: offset for name, offset, _ in table}

    # the publisher's manifest, and the check that these bytes are what it says
    digests = ctx.hash_chunks(blob, chunk_bytes)
    manifest = ctx.make_manifest(blob.numel(), chunk_bytes, digests.clone(), bytes(ctx.merkle_root(digests).cpu().numpy()))
    verdict, changed = binding.new_result(device), torch.zeros(digests.shape[0], dtype=torch.int64, device=device)
    ctx.verify_manifest(blob, manifest, verdict, changed)
    if not binding.read_result(verdict)["root_ok"]:
        raise RuntimeError("the weights are not what the manifest says")
    tree = ctx.tree_build(digests)

    weights, up = tensor_view(blob, table, embedding, shapes), tensor_view(blob, table, projection, shapes)
    norm_w = None if norm_weight is None else tensor_view(blob, table, norm_weight, shapes)
    rows, h = weights.shape
    generator = torch.Generator(device=device)
    generator.manual_seed(seed)
    tokens = torch.randint(0, rows, (n_tokens,), generator=generator, device=device)
    target = torch.randn(n_tokens, up.shape[0], generator=generator, device=device, dtype=torch.float32)
    norms, dirty_sets, losses, norm = binding.new_norm_result(device), [], [], []
    trained = [(embedding, weights), (projection, up)] + ([] if norm_w is None else [(norm_weight, norm_w)])

    def chunks_of_tensor(name: str, tensor: torch.Tensor) -> torch.Tensor:
        return chunks_of(torch.tensor([offset_of[name]], device=device), 2 * tensor.numel(), chunk_bytes)

    if optimizer != "sgd":
        # the trained tensors as a set in the file's bytes, their gradients back to back, and the state
        counts = [tensor.numel() for _, tensor in trained]
        starts = [sum(counts[:k]) for k in range(len(counts))]
        in_bytes = lambda values: torch.tensor([2 * v for v in values], dtype=torch.int64, device=device)  # noqa: E731
        offsets = torch.tensor([offset_of[name] for name, _ in trained], dtype=torch.int64, device=device)
        lengths, grad_offsets = in_bytes(counts), in_bytes(starts)
        grads = torch.empty(sum(counts), dtype=torch.bfloat16, device=device)
        d_table, *d_rest = (grads[a:a + n].view(tensor.shape) for a, n, (_, tensor) in zip(starts, counts, trained))
        state = binding.adamw_state(counts, device, bits=8 if optimizer == "adamw8" else 32)
    for _ in range(steps):
        s = forward(ctx, weights, up, norm_w, tokens, target)
        losses.append(float(s["loss"]))
        d_up, d_hidden, d_norm = backward(ctx, s, up, norm_w)
        if optimizer != "sgd":
            ctx.embedding_grad(d_hidden, tokens, rows, scale=math.sqrt(h), out=d_table)
            for to, gradient in zip(d_rest, (d_up, d_norm)):
                to.copy_(gradient)
            ctx.grad_norm(grads, grad_offsets, lengths, norms)
            ctx.adamw_step(blob, offsets, lengths, grads, grad_offsets, **state, lr=1e-3 * lr, norm=norms, max_norm=max_norm,
                           stochastic=True, seed=seed, dtype=torch.bfloat16)
            r = binding.read_norm_result(norms)
            norm.append(r["norm"])
            if r["n_nonfinite"]:
                continue                                 # the step has changed nothing
            dirty = torch.unique(torch.cat([chunks_of_tensor(name, tensor) for name, tensor in trained]))
        else:
            touched, d_rows, count = ctx.embedding_grad_rows(d_hidden, tokens, rows, scale=math.sqrt(h))
            base, offsets, lengths, types = binding.tensor_ranges([d_rows, d_up] + ([] if d_norm is None else [d_norm]))
            ctx.grad_clip(base, offsets, lengths, max_norm, norms, types=types)
            r = binding.read_norm_result(norms)
            norm.append(r["norm"])
            if r["n_nonfinite"]:
                continue                                 # an overflow somewhere: this step changes nothing
            n = int(count)
            weights.index_add_(0, touched[:n], d_rows[:n], alpha=-lr)      # distinct rows: no order to speak of
            up.add_(d_up, alpha=-lr)
            if norm_w is not None:
                norm_w.add_(d_norm, alpha=-lr)
            dirty = torch.unique(torch.cat([chunks_of(offset_of[embedding] + touched[:n] * (2 * h), 2 * h, chunk_bytes)]
                                           + [chunks_of_tensor(name, tensor) for name, tensor in trained[1:]]))
        ctx.tree_update(blob, chunk_bytes, dirty, tree)
        dirty_sets.append(dirty)

    # the retained tree against everything hashed anew, and what the manifest now says has changed
    fresh = ctx.merkle_root(ctx.hash_chunks(blob, chunk_bytes))
    ctx.verify_manifest(blob, manifest, verdict, changed)
    after = binding.read_result(verdict)
    return {"losses": losses, "norms": norm, "root": bytes(tree[-1].cpu().numpy()), "fresh_root": bytes(fresh.cpu().numpy()),
            "chunks": digests.shape[0], "dirty": torch.unique(torch.cat(dirty_sets)).tolist() if dirty_sets else [],
            "changed": changed[:after["n_mismatch"]].tolist(), "root_ok": after["root_ok"]}


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--layers", choices=("tiny", "gpt"), default="tiny")
    parser.add_argument("--steps", type=int, default=3)
    parser.add_argument("--norm", action="store_true", help="a root-mean-square norm before the projection")
    parser.add_argument("--optimizer", choices=("sgd", "adamw", "adamw8"), default="sgd")
    a = parser.parse_args()
    with binding.Context() as ctx:
        if a.layers == "tiny":
            r = run(ctx, inputs.tiny_tensors(), "embed.weight", "layers.0.up.weight", 4096, a.steps, 24,
                    norm_weight="layers.0.norm.weight" if a.norm else None, optimizer=a.optimizer)
        else:
            r = run(ctx, inputs.gpt_1p3b_tensors(), "wte.weight", "h.0.mlp.fc.weight", 1 << 20, a.steps, 2048,
                    norm_weight="h.0.ln_2.weight" if a.norm else None, optimizer=a.optimizer)
    print(f"losses {r['losses']}  gradient norms {r['norms']}")
    print(f"root {r['root'].hex()}: {'equal to' if r['root'] == r['fresh_root'] else 'NOT'} a full re-hash; "
          f"{len(r['changed'])} of {r['chunks']} chunks differ from the manifest, {len(r['dirty'])} were re-hashed")


if __name__ == "__main__":
    main()
