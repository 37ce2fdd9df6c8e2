"""Trains a small stack of 8-bit dense blocks (paper_1404_5997_amd/dense8.py) on rows around class centres, then serves single rows with it.

    python train_dense8.py [--rows 1024 --width 1024 --hidden 4096 --blocks 4 --classes 125 --steps 200 --rate 0.02 --dtype bf16]
                           [--loss softmax --max-norm 1.0]
"""
import argparse

import torch        # first: the library uses the HIP runtime that torch brings

from paper_1404_5997_amd.dense8 import Dense8Stack


def at_least_one(text):
    n = int(text)
    if n < 1:
        raise argparse.ArgumentTypeError("%d is less than one" % n)
    return n


def above_zero(text):
    v = float(text)
    if not v > 0.0:
        raise argparse.ArgumentTypeError("%s is not greater than zero" % text)
    return v


def main(argv=None):
    ap = argparse.ArgumentParser(description="Trains a small stack of 8-bit dense blocks and serves single rows with it.")
    for name, default in (("rows", 1024), ("width", 1024), ("hidden", 4096), ("classes", 125), ("steps", 200)):
        ap.add_argument("--" + name, type=at_least_one, default=default)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--rate", type=float, default=0.02)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    ap.add_argument("--loss", choices=("logistic", "softmax"), default="logistic")
    ap.add_argument("--max-norm", type=above_zero, default=None, help="bound on the norm of a step's gradients")
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    net = Dense8Stack(a.rows, a.width, a.hidden, a.blocks, a.classes, a.dtype, loss=a.loss, max_norm=a.max_norm)
    net.init(0)
    centres = torch.randn((a.classes, a.width), generator=g, device="cuda")
    for k in range(a.steps):
        labels = torch.randint(0, a.classes, (a.rows,), generator=g, device="cuda", dtype=torch.int32)
        x = (centres[labels.long()] + 0.5 * torch.randn((a.rows, a.width), generator=g, device="cuda")).to(net.tdt)
        net.step(x, labels, eps=a.rate)
        if k % 25 == 0 or k == a.steps - 1:
            norm = "" if a.max_norm is None else ", gradients %.4f" % net.grad_norm.item()
            print("step %d: loss %.4f%s" % (k, net.loss.mean().item(), norm), flush=True)
    whole = a.rows * ((a.blocks + 1) * 2 * a.width + a.blocks * a.hidden) * net.x.element_size()     # (the last norm has no hidden rows behind it)
    print("kept for the backward pass: %.1f MB (in storage type it would be %.1f)" % (net.checkpoint_bytes() / 1e6, whole / 1e6))
    one = Dense8Stack(1, a.width, a.hidden, a.blocks, a.classes, a.dtype)      # a served row: the trained weights, one row at a time
    one.params.copy_(net.params)
    one.pack_weights()
    served = min(64, a.rows)
    right = sum(int(one.forward(x[i:i + 1]).argmax()) == int(labels[i]) for i in range(served))
    print("single rows: %d of %d right" % (right, served))


if __name__ == "__main__":
    main()
