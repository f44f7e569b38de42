"""Fine-tuning steps on verified weights: verify, look up, differentiate, clip, update, re-verify what changed.

    python examples/verified_finetune_step.py [--layers gpt] [--steps 3]

The weights are one byte blob in device memory (a weight file: header, tensor index, bf16 tensors back to back) that has
been verified against its manifest; every tensor used below is a view into those bytes.  A step trains two of them,
the embedding table and one projection, on a regression target:

    hidden = sqrt(h) * table[tokens]        ctx.embedding
    y      = hidden @ up^T                  (library product)
    rows, d_table = gradient of the lookup  ctx.embedding_grad_rows: the touched rows only
    norm over both gradients, clipping      ctx.grad_clip
    table[rows] -= lr * d_table, up -= ...  in place, in the verified bytes
    the chunks those bytes lie in           ctx.tree_update -> new root

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


def run(ctx: binding.Context, tensors, embedding: str, projection: str, chunk_bytes: int, steps: int, n_tokens: int,
        lr: float = 2.0, max_norm: float = 0.02, seed: int = 1) -> dict:
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
    rows, h = weights.shape
    generator = torch.Generator(device=device)
    generator.manual_seed(seed)
    tokens = torch.randint(0, rows, (n_tokens,), generator=generator, device=device)
    target = torch.randn(n_tokens, up.shape[0], generator=generator, device=device, dtype=torch.float32)
    norms, dirty_sets, losses, norm = binding.new_norm_result(device), [], [], []
    for _ in range(steps):
        hidden = ctx.embedding(weights, tokens, scale=math.sqrt(h))
        error = (hidden @ up.t()).float() - target
        losses.append(float(error.square().mean()))
        d_y = (error * (2.0 / error.numel())).to(torch.bfloat16)
        d_up = d_y.t() @ hidden
        touched, d_rows, count = ctx.embedding_grad_rows(d_y @ up, tokens, rows, scale=math.sqrt(h))
        base, offsets, lengths, types = binding.tensor_ranges([d_rows, d_up])
        ctx.grad_clip(base, offsets, lengths, max_norm, norms, types=types)
        r = binding.read_norm_result(norms)
        norm.append(r["norm"])
        if r["n_nonfinite"]:
            continue                                     # an overflow somewhere: this step changes nothing
        n = int(count)
        weights.index_add_(0, touched[:n], d_rows[:n], alpha=-lr)      # distinct rows: no order to speak of
        up.add_(d_up, alpha=-lr)
        dirty = torch.unique(torch.cat([
            chunks_of(offset_of[embedding] + touched[:n] * (2 * h), 2 * h, chunk_bytes),
            chunks_of(torch.tensor([offset_of[projection]], device=device), 2 * up.numel(), chunk_bytes)]))
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
    a = parser.parse_args()
    with binding.Context() as ctx:
        if a.layers == "tiny":
            r = run(ctx, inputs.tiny_tensors(), "embed.weight", "layers.0.up.weight", 4096, a.steps, 24)
        else:
            r = run(ctx, inputs.gpt_1p3b_tensors(), "wte.weight", "h.0.mlp.fc.weight", 1 << 20, a.steps, 2048)
    print(f"losses {r['losses']}  gradient norms {r['norms']}")
    print(f"root {r['root'].hex()}: {'equal to' if r['root'] == r['fresh_root'] else 'NOT'} a full re-hash; "
          f"{len(r['changed'])} of {r['chunks']} chunks differ from the manifest, {len(r['dirty'])} were re-hashed")


if __name__ == "__main__":
    main()
