"""A binary MLP that classifies hidden states of a language model (synthetic ones).

The 8-bit front end takes the bf16 hidden states to the packed +-1 words that a
BMLP reads, all on the device and on one stream:

  bmlp_quantize_rows   the projection's channels to 8 bits, once
  bmlp_int8_matmul     sums of a few hundred rows, for thresholds at their medians
  bmlp_norm_quantize   residual + hidden state, RMS norm, to 8 bits
  bmlp_int8_sign       the projection's signs against the thresholds, packed

then bmlp_train / bmlp_predict run on the words; at the end one hidden state at
a time is classified, as a server would.

  python examples/hidden_states.py [--n 20000 --dim 1024 --width 2048 --epochs 10]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2412_00119_gb300 import bmlp as B  # noqa: E402


def hidden_states(n, dim, classes, gen):
    """n rows (hidden state, residual) around a direction per class, with rows of different
    sizes and a few channels much larger than the others."""
    dev = "cuda"
    centre = torch.randn((classes, dim), generator=torch.Generator(dev).manual_seed(1), device=dev)
    large = torch.rand((dim,), generator=torch.Generator(dev).manual_seed(2), device=dev) < 1 / 128
    y = torch.randint(0, classes, (n,), generator=gen, device=dev, dtype=torch.int32)
    x = 0.25 * centre[y.long()] + torch.randn((n, dim), generator=gen, device=dev)
    x *= torch.where(large, 16.0, 1.0) * torch.exp(0.5 * torch.randn((n, 1), generator=gen, device=dev))
    res = 0.5 * torch.randn((n, dim), generator=gen, device=dev) * x.abs().mean(1, keepdim=True)
    return x.bfloat16(), res.bfloat16(), y


class FrontEnd:
    """Norm, 8-bit projection and thresholds of a fixed layer dim -> width."""

    def __init__(self, dim, width, gain, gen):
        w = torch.randn((width, dim), generator=gen, device="cuda") / dim ** 0.5
        self.gain, self.width = gain, width
        self.w = torch.empty((width, dim), dtype=torch.int8, device="cuda")
        self.w_scale = torch.empty((width,), device="cuda")
        B.bmlp_quantize_rows(w.bfloat16(), self.w, self.w_scale)
        self.threshold = None

    def codes(self, x, res):
        q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
        scale = torch.empty((x.shape[0],), device="cuda")
        B.bmlp_norm_quantize(x, self.gain, q, scale, res=res)
        return q, scale

    def calibrate(self, x, res):
        """Thresholds at the medians of the sums of these rows: bits that are half ones."""
        q, _ = self.codes(x, res)
        sums = torch.empty((x.shape[0], self.width), dtype=torch.int32, device="cuda")
        B.bmlp_int8_matmul(q, self.w, sums)
        self.threshold = sums.median(0).values.to(torch.int32)

    def words(self, x, res):
        q, _ = self.codes(x, res)
        out = torch.empty((x.shape[0], (self.width + 63) // 64), dtype=torch.int64, device="cuda")
        B.bmlp_int8_sign(q, self.w, out, self.threshold)
        return out

    def project(self, x, res):
        """The projection itself, fp32 (what the signs are taken of)."""
        q, scale = self.codes(x, res)
        out = torch.empty((x.shape[0], self.width), device="cuda")
        B.bmlp_int8_matmul(q, self.w, out, scale, self.w_scale)
        return out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--n", type=int, default=20000)
    ap.add_argument("--dim", type=int, default=1024)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--classes", type=int, default=10)
    ap.add_argument("--epochs", type=int, default=10)
    a = ap.parse_args(argv)
    gen = torch.Generator("cuda").manual_seed(3)
    x, res, y = hidden_states(a.n, a.dim, a.classes, gen)
    xt, rt, yt = hidden_states(max(1, a.n // 5), a.dim, a.classes, gen)
    gain = (1 + 0.1 * torch.randn((a.dim,), generator=gen, device="cuda")).bfloat16()
    front = FrontEnd(a.dim, a.width, gain, gen)
    front.calibrate(x[:512], res[:512])
    # the 8-bit projection beside the one in fp32
    h = x[:64].float() + res[:64].float()
    exact = h / h.square().mean(1, keepdim=True).sqrt() * gain.float() @ (front.w.float() * front.w_scale[:, None]).t()
    err = (front.project(x[:64], res[:64]) - exact).norm() / exact.norm()
    model = B.BMLP([a.width, 255, 255], a.classes, seed=5)
    words, test = front.words(x, res), front.words(xt, rt)
    labels = torch.empty((len(yt),), dtype=torch.int32, device="cuda")
    for epoch in range(a.epochs):
        errors = model.train(words, y, epoch_end=True, count_errors=True)
    model.predict(test, labels)
    accuracy = (labels == yt).float().mean().item()
    # one hidden state at a time gives the same labels
    one = torch.empty((1,), dtype=torch.int32, device="cuda")
    same = True
    for i in range(min(20, len(yt))):
        model.predict(front.words(xt[i:i + 1], rt[i:i + 1]), one)
        same = same and one.item() == labels[i].item()
    model.close()
    print("8-bit projection: relative error %.4f; training errors in the last epoch %d of %d; "
          "test accuracy %.3f; one at a time %s" % (err, errors, a.n, accuracy, "the same" if same else "different"))
    return dict(error=err.item(), accuracy=accuracy, same=same, words=words, y=y, test=test, labels=labels, errors=errors)


if __name__ == "__main__":
    main()
