"""Training a stack of residual blocks with knowledge-guided freezing, every step of it on the library's kernels.

    python examples/train_frozen_blocks.py [--steps 200] [--blocks 6] [--hidden 256] [--eight-bit] [--gated] [--muon]

Each block is norm -> linear + gelu -> linear, or with --gated norm -> gated feed-forward, added to the residual stream through a gate.
A step runs

    forward    egeria_linear_forward (bias and activation in its epilogue) or egeria_gated_forward, egeria_norm_forward (a block's output
               norm, its gate, the addition and the next block's input norm in one pass)
    freezing   egeria_plasticity_evaluate on the blocks' outputs against those of a reference model, every few steps
    backward   egeria_norm_backward, egeria_linear_backward or egeria_gated_backward, from the last block down to the first that still
               trains
    update     egeria_adamw_step with the freeze mask as the evaluation left it on the device; with --muon the matrices by
               egeria_muon_step under the same mask

The mask is read back once per evaluation, to stop the backward pass at the frozen prefix; the optimizer needs no read.
The task is synthetic: the outputs of a fixed random network of the same shape.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

from paper_2201_06227_b200 import binding as eg  # noqa: E402
from paper_2201_06227_b200 import ops  # noqa: E402

DTYPE = torch.bfloat16


def gated_width(hidden):
    """The usual 8/3 of the width, rounded up to a multiple of 64."""
    return -(-8 * hidden // 192) * 64


class Blocks:
    """The parameters of a stack of blocks and its forward and backward pass."""

    NAMES = ("w1", "b1", "w2", "b2", "w_post", "b_post", "gate", "w_pre", "b_pre")   # w_pre, b_pre: of the norm behind the block
    GATED = ("w_gate", "w_up", "w_down", "w_post", "b_post", "gate", "w_pre", "b_pre")

    def __init__(self, blocks, hidden, handle, seed, device, gated=False):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(*shape, generator=g, device=device) * scale).to(DTYPE)

        one, zero = (lambda: torch.ones(hidden, dtype=DTYPE, device=device)), (lambda: torch.zeros(hidden, dtype=DTYPE, device=device))
        self.ops, self.hidden, self.gated, self.names = handle, hidden, gated, self.GATED if gated else self.NAMES
        wide = gated_width(hidden)
        self.params = [dict(w_gate=normal(wide, hidden, scale=hidden ** -0.5), w_up=normal(wide, hidden, scale=hidden ** -0.5),
                            w_down=normal(hidden, wide, scale=wide ** -0.5), w_post=one(), b_post=zero(),
                            gate=torch.full((hidden,), 0.5, dtype=DTYPE, device=device), w_pre=one(), b_pre=zero()) for _ in range(blocks)] if gated else \
                      [dict(w1=normal(4 * hidden, hidden, scale=hidden ** -0.5), b1=normal(4 * hidden, scale=0.02),
                            w2=normal(hidden, 4 * hidden, scale=(4 * hidden) ** -0.5), b2=normal(hidden, scale=0.02), w_post=one(), b_post=zero(),
                            gate=torch.full((hidden,), 0.5, dtype=DTYPE, device=device), w_pre=one(), b_pre=zero()) for _ in range(blocks)]

    def copy_from(self, other):
        for mine, theirs in zip(self.params, other.params):
            for k in self.names:
                mine[k].copy_(theirs[k])

    def forward(self, x, first_kept=0):
        """(last h, what the backward pass of blocks first_kept.. needs, the stream after every block)."""
        _, h, _ = self.ops.egeria_norm_forward(x, x, post=False, alpha=0.0)       # N(x) alone: the stream is its own branch
        kept, outputs = [], []
        for i, p in enumerate(self.params):
            keep = i >= first_kept
            if self.gated:
                f = self.ops.egeria_gated_forward(h, p["w_gate"], p["w_up"], p["w_down"], save=keep)
                f, a, z = f if keep else (f, None, None)      # a, z: the two projections
            else:
                a = self.ops.egeria_linear_forward(h, p["w1"], bias=p["b1"], act="gelu", save_z=keep)
                a, z = a if keep else (a, None)
                f = self.ops.egeria_linear_forward(a, p["w2"], bias=p["b2"])
            x, h_next, stats = self.ops.egeria_norm_forward(x, f, gate=p["gate"], w_post=p["w_post"], b_post=p["b_post"], w_pre=p["w_pre"],
                                                            b_pre=p["b_pre"])
            kept.append((h, a, z, f, x, stats) if keep else None)
            outputs.append(x)
            h = h_next
        return h, kept, outputs

    def backward(self, dh, kept, first, grads):
        """Writes the gradients of blocks first.. into `grads`, from the gradient of the last h."""
        dx = torch.zeros_like(dh)
        for i in range(len(self.params) - 1, first - 1, -1):
            p, g = self.params[i], grads[i]
            h, a, z, f, y, stats = kept[i]
            n = self.ops.egeria_norm_backward(dx, dh, y, f, stats, gate=p["gate"], w_post=p["w_post"], b_post=p["b_post"], w_pre=p["w_pre"],
                                              b_pre=p["b_pre"])
            if self.gated:
                b = self.ops.egeria_gated_backward(n["df"], h, p["w_gate"], p["w_up"], p["w_down"], a, z, need_dx=i > first)
                dh, own = b["dx"], dict(w_gate=b["dw_gate"], w_up=b["dw_up"], w_down=b["dw_down"])
            else:
                # the second product's dx is the first one's dz: the activation's slope goes into its epilogue
                dz, dw2, db2 = self.ops.egeria_linear_backward(n["df"], a, p["w2"], z_in=z, act_in="gelu")
                dh, dw1, db1 = self.ops.egeria_linear_backward(dz, h, p["w1"], need_dx=i > first)
                own = dict(w1=dw1, b1=db1, w2=dw2, b2=db2)
            dx = n["dx"]
            for k, v in dict(own, w_post=n["dw_post"], b_post=n["db_post"], gate=n["dgate"], w_pre=n["dw_pre"], b_pre=n["db_pre"]).items():
                g[k].copy_(v)


def train(blocks=6, hidden=256, batch=32, seq=16, steps=200, every=4, window=4, tolerance=2e-4, lr=2e-3, bits=32, seed=0, device="cuda", gated=False, muon=False,
          log=print):
    """Trains and returns (losses, modules frozen at the end, the model, its parameters at the time each block froze)."""
    rows = batch * seq
    handle = ops.Ops(max(ops.egeria_linear_workspace_bytes(rows, hidden, 4 * hidden), ops.egeria_linear_workspace_bytes(rows, 4 * hidden, hidden),
                         ops.egeria_gated_workspace_bytes(rows, hidden, gated_width(hidden), hidden), ops.egeria_norm_workspace_bytes(rows, hidden)), device)
    model, reference, teacher = (Blocks(blocks, hidden, handle, seed + k, device, gated) for k in (1, 2, 3))
    reference.copy_from(model)

    matrix = ("w1", "w2", "w_gate", "w_up", "w_down")
    grads = [{k: torch.zeros_like(v) for k, v in p.items()} for p in model.params]
    matrices = None
    if muon:                                             # the matrices; AdamW keeps the vectors
        tensors = [(i, k) for i in range(blocks) for k in model.names if k in matrix]
        params = [model.params[i][k] for i, k in tensors]
        matrices = ops.Muon(params, [grads[i][k] for i, k in tensors], [torch.zeros(p.shape, device=device) for p in params],
                            masters=[p.float() for p in params], weight_decay=0.01, scale="rms", modules=[i for i, _ in tensors])
    tensors = [(i, k) for i in range(blocks) for k in model.names if not (muon and k in matrix)]
    params = [model.params[i][k] for i, k in tensors]
    masters = [p.float() for p in params]
    steps_taken = torch.zeros(len(params), dtype=torch.int32, device=device)
    if bits == 8:
        scales = [torch.zeros(-(-p.numel() // ops.ADAMW_BLOCK), device=device) for p in params]
        moments = dict(exp_avg=[torch.zeros(p.shape, dtype=torch.int8, device=device) for p in params],
                       exp_avg_sq=[torch.zeros(p.shape, dtype=torch.uint8, device=device) for p in params],
                       m_scales=scales, v_scales=[s.clone() for s in scales])
    else:
        moments = dict(exp_avg=[torch.zeros_like(m) for m in masters], exp_avg_sq=[torch.zeros_like(m) for m in masters])
    adamw = ops.AdamW(params, [grads[i][k] for i, k in tensors], steps=steps_taken, masters=masters,
                      weight_decay=[0.01 if k in matrix else 0.0 for _, k in tensors], modules=[i for i, _ in tensors], **moments)
    plasticity = eg.Context([seq * hidden] * blocks, batch, window, tolerance, eg.FLAG_FRONTMOST, device=device)

    g = torch.Generator(device=device)
    g.manual_seed(seed)
    mask = torch.zeros(blocks, dtype=torch.uint8, device=device)
    frozen, at_freeze, losses = 0, {}, []
    for step in range(steps):
        x = torch.randn(rows, hidden, generator=g, device=device).to(DTYPE)
        target = teacher.forward(x, first_kept=blocks)[0]
        h, kept, outputs = model.forward(x, first_kept=frozen)
        error = h.float() - target.float()
        losses.append((error * error).mean())
        if step % every == 0:
            if step % (8 * every) == 0:
                reference.copy_from(model)          # the reference follows the model at a distance
            ref = reference.forward(x, first_kept=blocks)[2]
            _, _, mask = plasticity.egeria_plasticity_evaluate([o.view(batch, -1) for o in outputs], [o.view(batch, -1) for o in ref])
            now = int(mask.sum())                   # the one read back: how far down the backward pass has to go
            for i in range(frozen, now):
                at_freeze[i] = {k: v.clone() for k, v in model.params[i].items()}
            if now != frozen:
                log(f"step {step}: {now} of {blocks} blocks frozen, loss {float(losses[-1]):.4f}")
            frozen = now
            if frozen == blocks:
                break
        model.backward((error * (2.0 / rows)).to(DTYPE), kept, frozen, grads)
        adamw.egeria_adamw_step(lr, frozen=mask)
        if matrices is not None:
            matrices.egeria_muon_step(lr, frozen=mask)
    plasticity.check_device_status()
    handle.check_device_status()
    adamw.check_device_status()
    if matrices is not None:
        matrices.check_device_status()
    return [float(v) for v in losses], frozen, model, at_freeze


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--steps", type=int, default=200)
    a.add_argument("--blocks", type=int, default=6)
    a.add_argument("--hidden", type=int, default=256)
    a.add_argument("--eight-bit", action="store_true", help="moments in 8 bits")
    a.add_argument("--gated", action="store_true", help="gated feed-forward blocks")
    a.add_argument("--muon", action="store_true", help="Muon for the matrices")
    a = a.parse_args()
    losses, frozen, _, _ = train(blocks=a.blocks, hidden=a.hidden, steps=a.steps, bits=8 if a.eight_bit else 32, gated=a.gated, muon=a.muon)
    print(f"{len(losses)} steps: loss {losses[0]:.4f} -> {losses[-1]:.4f}, {frozen} of {a.blocks} blocks frozen")


if __name__ == "__main__":
    main()
