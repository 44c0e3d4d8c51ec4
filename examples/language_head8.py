"""The end of a language model, trained and used for scoring with the 8-bit operators.

    h = x + residual;  y = rms_norm(h);  logits = y W^T;  log probabilities of the given tokens

The norm takes the residual's addition in and leaves its result packed, as the product's operand.  The gradient of
the log probabilities (and of the entropy, where it is wanted) leaves packed in rows and columns, as the operands of the two
gradient products.  The weight's update is its gradient orthogonalised by Newton-Schulz products.

    python examples/language_head8.py            trains on a synthetic task, then scores one token
"""
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for path in (ROOT, os.path.join(ROOT, "examples")):
    if path not in sys.path:
        sys.path.insert(0, path)

import paper_1501_06633_b200 as mx  # noqa: E402
from feed_forward8 import Linear8, columns_of, scales  # noqa: E402


class LanguageHead8:
    def __init__(self, width, vocabulary, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.width, self.vocabulary = width, vocabulary
        self.gamma = torch.ones(width, device="cuda")
        self.out = Linear8(vocabulary, width, gen)
        self.kept = None

    def logits(self, x, residual):
        """Logits of each token, and what the backward pass needs of the norm."""
        t, w = x.shape
        y, rstd, h = (mx.empty_packed(t, w), scales(mx.BLOCK_ROW, t, w)), torch.empty(t, device="cuda"), torch.empty_like(x)
        mx.rms_norm_fprop(mx.RmsNormDesc.make(t, w), x, self.gamma, residual=residual, sum=h, rstd=rstd, packed=y)
        z = torch.empty(t, self.vocabulary, dtype=torch.bfloat16, device="cuda")
        self.out.forward(*y, z)
        return z, (y, rstd, h)

    def forward(self, x, residual, tokens, top=0):
        """Log probabilities of `tokens`, entropies, and the `top` most likely tokens with theirs."""
        t, (z, norm) = x.shape[0], self.logits(x, residual)
        new = lambda *s: torch.empty(*s, device="cuda")
        logprob, lse, entropy = new(t), new(t), new(t)
        likely = dict(top_logprob=new(t, top), top_index=torch.empty(t, top, dtype=torch.int32, device="cuda")) if top else {}
        mx.logprob_fprop(mx.LogprobDesc.make(t, self.vocabulary, top=top), z, tokens, logprob=logprob, lse=lse, entropy=entropy, **likely)
        self.kept = (z, tokens, lse, entropy, norm)
        return logprob, entropy, likely

    def backward(self, dlogprob, dentropy=None, dsum=None):
        """Gradients by name from those of the log probabilities, the entropies and of what else reads the norm's sum."""
        z, tokens, lse, entropy, (y, rstd, h) = self.kept
        (t, w), v = h.shape, self.vocabulary
        row = mx.empty_packed(t, v, mx.DTYPE_E5M2), scales(mx.BLOCK_ROW, t, v)
        col = mx.empty_packed(t, v, mx.DTYPE_E5M2), scales(mx.BLOCK_COL, t, v)
        mx.logprob_bprop(mx.LogprobDesc.make(t, v), z, tokens, lse, dlogprob=dlogprob, entropy=entropy, dentropy=dentropy, row=row, col=col)
        grads = {"out": self.out.weight_gradient(*col, *columns_of(*y)), "logits": (row, col)}
        dy, dx = torch.empty_like(h), torch.empty_like(h)
        self.out.input_gradient(*row, dy)
        d = mx.RmsNormDesc.make(t, w)
        ws = torch.empty(max(16, mx.rms_norm_bprop_workspace(d)), dtype=torch.uint8, device="cuda")
        grads["gamma"] = torch.empty(w, device="cuda")
        mx.rms_norm_bprop(d, dy, h, self.gamma, rstd, dx, grads["gamma"], ws, dsum=dsum)
        grads["y"], grads["x"] = dy, dx                      # x and the residual have the same gradient
        return grads

    def update(self, grads, rate):
        """The weight moves along its orthogonalised gradient, gamma along its own."""
        v, w = self.vocabulary, self.width
        d = mx.OrthoDesc.make(v, w, x_type=mx.DTYPE_F32)
        step = torch.empty(v, w, dtype=torch.bfloat16, device="cuda")
        mx.orthogonalise(d, grads["out"], step, torch.empty(mx.orthogonalise_workspace(d), dtype=torch.uint8, device="cuda"))
        self.out.master -= rate * step
        self.out.pack()
        self.gamma -= rate * grads["gamma"]
        return step


def main():
    torch.manual_seed(0)
    tokens, width, vocabulary = 2048, 512, 4000
    head = LanguageHead8(width, vocabulary, seed=1)
    x, residual = (torch.randn(tokens, width, device="cuda").to(torch.bfloat16) for _ in range(2))
    goal = LanguageHead8(width, vocabulary, seed=2).logits(x, residual)[0].float().argmax(1)
    for step in range(31):
        logprob, entropy, _ = head.forward(x, residual, goal)
        head.update(head.backward(torch.full((tokens,), -1.0 / tokens, device="cuda")), rate=0.05)
        if step % 5 == 0:
            print("step %2d  loss %.3f  entropy %.3f" % (step, -float(logprob.mean()), float(entropy.mean())))
    one = [t[:1].contiguous() for t in (x, residual, goal)]
    for _ in range(3):
        head.forward(*one, top=5)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(100):
        head.forward(*one, top=5)
    torch.cuda.synchronize()
    print("one token: %.1f us" % ((time.perf_counter() - t) * 1e4))
    assert mx.last_device_status() == mx.OK


if __name__ == "__main__":
    main()
