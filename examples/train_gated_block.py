"""Trains the feed-forward half of a gated DiT block, and a projection with
rotary positions over an image grid, to match a teacher's outputs.

One step runs the gated block's layers as they follow one another in a block,
forward and backward: the norms around the branch with the AdaLN vectors, the gated
feed-forward and the rotary positions (``paper_2609_32415_gb300.training``). With
--linear4 the projection runs through 4-bit products, with --bits the optimiser is
``training.AdamW`` with moments of so many bits.

    python examples/train_gated_block.py [--steps 60] [--linear4] [--bits 8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_32415_gb300 import api, training  # noqa: E402
from paper_2609_32415_gb300._lib import RA_ACT_SILU, RA_NORM_RMS  # noqa: E402


class Block(torch.nn.Module):
    """h -> (h', q): h' = h + gate N(ff(N(h))), q = rope(N(h') Wq)."""

    def __init__(self, C, F, H, pos, axes, err, seed, linear4=False):
        super().__init__()
        self.linear4 = linear4
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, k):
            w = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
            return torch.nn.Parameter(w.to(torch.bfloat16))

        self.w_gate, self.w_up, self.w_down, self.w_q = weight(F, C), weight(F, C), weight(C, F), weight(C, C)
        ones = torch.ones(C, device="cuda")
        self.pre_a, self.post_a, self.pre_b = (torch.nn.Parameter(ones.clone()) for _ in range(3))
        self.H, self.pos, self.axes, self.err = H, pos, axes, err

    def forward(self, h, mods):
        _, x = training.residual_norm(h, None, RA_NORM_RMS, RA_NORM_RMS, pre_w=self.pre_a, scale=mods["scale"],
                                      shift=mods["shift"], err_word=self.err)
        y = training.gated_feed_forward(x, self.w_gate, self.w_up, self.w_down, RA_ACT_SILU, self.err)
        h, x = training.residual_norm(h, y, RA_NORM_RMS, RA_NORM_RMS, gate=mods["gate"], post_w=self.post_a,
                                      pre_w=self.pre_b, err_word=self.err)
        q = training.linear4(x, self.w_q, err_word=self.err) if self.linear4 else x @ self.w_q.T
        q = q.unflatten(2, (self.H, -1)).transpose(1, 2)
        return h, training.rope_axes(q, self.pos, self.axes)


def train(steps=60, B=2, height=20, width=27, C=512, F=1408, H=8, lr=0.06, report=None, linear4=False, bits=None):
    """Returns the losses of all steps."""
    axes = (C // H // 2, C // H // 2)
    pos = torch.stack(torch.meshgrid(torch.arange(height), torch.arange(width), indexing="ij"), -1)
    pos = pos.reshape(-1, 2).float().cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    teacher, student = Block(C, F, H, pos, axes, err, 1), Block(C, F, H, pos, axes, err, 2, linear4)
    with torch.no_grad():  # a student on its way to the teacher
        for a, b in zip(student.parameters(), teacher.parameters()):
            a.copy_((0.5 * a.float() + 0.5 * b.float()).to(a.dtype))
    opt = torch.optim.Adam(student.parameters(), lr=lr * C ** -0.5) if bits is None else \
        training.AdamW(student.parameters(), lr=lr * C ** -0.5, weight_decay=0.0, bits=bits, max_norm=10.0)
    g = torch.Generator(device="cuda").manual_seed(3)
    losses = []
    for step in range(steps):
        h = torch.randn((B, height * width, C), generator=g, device="cuda").to(torch.bfloat16)
        mods = {k: 0.1 * torch.randn((B, C), generator=g, device="cuda") + (1.0 if k == "gate" else 0.0)
                for k in ("scale", "shift", "gate")}
        with torch.no_grad():
            want = teacher(h, mods)
        got = student(h, mods)
        loss = sum(((a.float() - b.float()) ** 2).mean() for a, b in zip(got, want))
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if report and (step % 10 == 0 or step + 1 == steps):
            report("step %3d  loss %.5f" % (step, float(losses[-1])))
    api.refadapt_check_error(err)
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--linear4", action="store_true")
    ap.add_argument("--bits", type=int, choices=(8, 32))
    args = ap.parse_args()
    train(args.steps, report=print, linear4=args.linear4, bits=args.bits)
