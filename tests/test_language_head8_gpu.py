"""A training step of the norm, the product, the log probabilities, their gradient and the update together, as the example
runs it: every result against its formula in 64 bits, from the values that the operator in front of it left.

Tolerances.  16-bit results: half a step, 2^-8 of the value, besides 2^-16 of the sum of magnitudes for a product's and a
norm's 32-bit sums.  Packed results: half a step of the 8-bit type.  The update: see test_orthogonalise_gpu.py."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import logprob_ref
import paper_1501_06633_b200 as mx
import train8_ref as ref
from packed_rows import near_rows
from test_orthogonalise_gpu import formula, near
from test_train8_gpu import bytes_of, down

pytestmark = pytest.mark.gpu
AT = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "language_head8.py")
spec = importlib.util.spec_from_file_location("language_head8", AT)
lh = importlib.util.module_from_spec(spec)
spec.loader.exec_module(lh)
HALF, SUMS = 2.0 ** -8, 2.0 ** -16


def value(q, s, form):
    return down(q) * ref.spread(ref.value_of(bytes_of(s)), form, *q.shape)


def transposed(q):
    return q.view(torch.uint8).t().contiguous().view(q.dtype)


def given(tokens, width, vocabulary, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, r, ds = (torch.randn(tokens, width, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    tok = torch.randint(0, vocabulary, (tokens,), device="cuda", generator=gen)
    tok[::5] = -1
    dlp, dh = (torch.randn(tokens, device="cuda", generator=gen) for _ in range(2))
    return x, r, ds, tok, dlp, dh


@pytest.mark.parametrize("tokens,width,vocabulary", [(1, 128, 500), (70, 200, 1000), (130, 512, 801), (300, 264, 3001)])
def test_a_step(tokens, width, vocabulary):
    head = lh.LanguageHead8(width, vocabulary, seed=1)
    head.gamma += 0.1 * torch.randn(width, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    x, r, ds, tok, dlp, dh = given(tokens, width, vocabulary, 3)
    logprob, entropy, likely = head.forward(x, r, tok, top=5)
    z, _, lse, _, ((q, s), rstd, h) = head.kept
    grads = head.backward(dlp, dh, ds)
    step = head.update(grads, rate=0.0)
    assert mx.last_device_status() == mx.OK
    # norm
    full = down(x) + down(r)
    assert np.all(np.abs(down(h) - full) <= HALF * np.abs(full))
    wr = 1 / np.sqrt((full ** 2).mean(1) + 1e-6)
    y = full * wr[:, None] * down(head.gamma)
    near_rows(q, s, y, SUMS * np.abs(y), "e4m3")
    # product
    yq, w = value(q, s, "row"), value(head.out.q, head.out.s, "tile")
    want, size = yq @ w.T, np.abs(yq) @ np.abs(w).T
    assert np.all(np.abs(down(z) - want) <= HALF * np.abs(want) + SUMS * size)
    # log probabilities of those logits
    t64 = tok.cpu().numpy()
    l, lp, e, tlp, idx, a1, a2 = logprob_ref.forward(down(z), 1.0, t64, 5)
    for got, ref64 in ((lse, l), (logprob, lp), (entropy, e), (likely["top_logprob"], tlp)):
        assert np.all(np.abs(down(got) - ref64) <= SUMS * (1 + np.abs(ref64)))
    np.testing.assert_array_equal(likely["top_index"].cpu().numpy(), idx)
    # their gradient, packed
    dz, tol = logprob_ref.gradient(down(z), 1.0, t64, down(lse), down(dlp), down(entropy), down(dh))
    row, col = grads["logits"]
    near_rows(*row, dz, tol, "e5m2")
    near_rows(transposed(col[0]), col[1], dz.T, tol.T, "e5m2")
    # the products behind it
    g, gc = value(*row, "row"), value(*col, "col")
    want, size = g @ w, np.abs(g) @ np.abs(w)
    assert np.all(np.abs(down(grads["y"]) - want) <= HALF * np.abs(want) + SUMS * size)
    yc, ys = ref.pack(yq, "col", "e4m3")
    yc = yc * ref.spread(ref.value_of(ys), "col", tokens, width)
    want, size = gc.T @ yc, np.abs(gc).T @ np.abs(yc)
    assert np.all(np.abs(down(grads["out"]) - want) <= SUMS * size)
    # the norm's gradient
    dy, hh = down(grads["y"]), down(h) * down(rstd)[:, None]
    e1 = dy * down(head.gamma)
    inner, size = (e1 * hh).mean(1, keepdims=True), np.abs(e1 * hh).mean(1, keepdims=True)
    want = down(rstd)[:, None] * (e1 - hh * inner) + down(ds)
    assert np.all(np.abs(down(grads["x"]) - want) <= HALF * np.abs(want) + SUMS * (down(rstd)[:, None] * (np.abs(e1) + np.abs(hh) * size) + np.abs(down(ds))))
    assert np.all(np.abs(down(grads["gamma"]) - (dy * hh).sum(0)) <= SUMS * np.abs(dy * hh).sum(0) + 1e-30)
    # the update
    near(step[None], formula(grads["out"][None], 5))


def test_steps_captured_and_run_again():
    """Two steps in a graph give what two steps without it give, whatever ran before."""
    tokens, width, vocabulary = 96, 256, 700
    x, r, ds, tok, dlp, dh = given(tokens, width, vocabulary, 5)
    results = []
    for captured in (False, True):
        head = lh.LanguageHead8(width, vocabulary, seed=4)
        start = head.out.master.clone()

        def two():
            for _ in range(2):
                head.forward(x, r, tok, top=3)
                head.update(head.backward(dlp, dh, ds), rate=1e-3)

        two()
        if captured:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                two()
        head.out.master.copy_(start)
        head.gamma.fill_(1.0)
        head.out.pack()
        torch.cuda.synchronize()
        graph.replay() if captured else two()
        torch.cuda.synchronize()
        results.append((head.out.master.clone(), head.gamma.clone()))
    assert mx.last_device_status() == mx.OK
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])


def test_the_example_runs(capsys, monkeypatch):
    lh.main()
    assert "one token" in capsys.readouterr().out


def test_both_ways_of_marshalling_make_the_same_calls(monkeypatch):
    """With the marshalling module, and with every call checked in Python."""
    from paper_1501_06633_b200 import train8
    x, r, ds, tok, dlp, dh = given(40, 136, 300, 6)
    got = []
    assert train8._library() and train8._plain is not train8._NoPlain, "the marshalling module is not built"
    for plain in (train8._plain, train8._NoPlain):
        monkeypatch.setattr(train8, "_plain", plain)
        head, before = lh.LanguageHead8(136, 300, seed=2), mx.launch_count()
        lp, h, likely = head.forward(x, r, tok, top=2)
        grads = head.backward(dlp, dh, ds)
        got.append(([lp, h, likely["top_index"], grads["out"], grads["x"], grads["gamma"], head.update(grads, 0.1)], mx.launch_count() - before))
    assert got[0][1] == got[1][1] and all(torch.equal(a, b) for a, b in zip(got[0][0], got[1][0]))


def test_the_marshalling_module_lets_other_threads_run():
    """The interpreter's lock is released around the library's calls: in their place stands the function that tells whether
    this thread holds it."""
    import ctypes
    from paper_1501_06633_b200 import train8
    lib, plain = train8._library(), train8._plain
    assert plain is not train8._NoPlain, "the marshalling module is not built"
    names = ("rms_norm_fprop", "rms_norm_bprop", "logprob_fprop", "logprob_bprop")
    held = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    x, v = torch.zeros(4, 128, device="cuda"), torch.zeros(4, device="cuda")
    tok, none = torch.zeros(4, dtype=torch.int64, device="cuda"), (None, None)
    rms, lp = mx.RmsNormDesc.make(4, 128, x_type=mx.DTYPE_F32), mx.LogprobDesc.make(4, 128, x_type=mx.DTYPE_F32)
    calls = {"rms_norm_fprop": (rms, x, None, None, None, x, v, *none, *none, None), "rms_norm_bprop": (rms, x, x, None, None, v, None, x, None, None, None),
             "logprob_fprop": (lp, x, tok, v, v, v, None, None, None), "logprob_bprop": (lp, x, tok, v, v, None, None, x, *none, *none, None)}
    try:
        plain.bind_more(*[held] * 4)
        got = {n: getattr(plain, n)(*calls[n]) for n in names}
    finally:
        plain.bind_more(*(ctypes.cast(getattr(lib, "maxdnn_" + n), ctypes.c_void_p).value for n in names))
    assert got == {n: 0 for n in names}          # (1: held, -1: the call was not plain)


@pytest.mark.parametrize("code", [6, 9, -1])
def test_types_that_do_not_exist(code):
    x, r, g = torch.zeros(4, 128, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(128, device="cuda")
    f, e8 = mx.DTYPE_F32, lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    refused = pytest.raises((TypeError, ValueError, mx.MaxdnnError))
    with refused:
        mx.rms_norm_fprop(mx.RmsNormDesc.make(4, 128, x_type=f, w_type=code), x, g, y=x)
    with refused:
        mx.rms_norm_fprop(mx.RmsNormDesc.make(4, 128, x_type=f, q_type=code), x, packed=(e8(4, 128), e8(1, 4)))
    with refused:
        mx.rms_norm_bprop(mx.RmsNormDesc.make(4, 128, x_type=code, y_type=f), x, x, None, r, torch.empty_like(x))
    with refused:
        mx.logprob_fprop(mx.LogprobDesc.make(4, 128, x_type=code), x, tok, r)
    with refused:
        mx.logprob_fprop(mx.LogprobDesc.make(4, 128, x_type=f, target_type=code), x, tok, r)
    with refused:
        mx.orthogonalise(mx.OrthoDesc.make(4, 128, x_type=code), x, torch.empty(4, 128, dtype=torch.bfloat16, device="cuda"), e8(1 << 20))
    for bad in (dict(x=x[:, :100]), dict(x=x.half()), dict(x=x.cpu()), dict(logprob=torch.empty(5, device="cuda")), dict(target=tok.int())):
        with refused:
            mx.logprob_fprop(mx.LogprobDesc.make(4, 128, x_type=f), **{**dict(x=x, target=tok, logprob=r), **bad})
    with refused:
        mx.rms_norm_bprop(mx.RmsNormDesc.make(4, 128, x_type=f), x, x, None, r, torch.empty_like(x), g, e8(4))      # a workspace too small
    with refused:
        mx.orthogonalise(mx.OrthoDesc.make(4, 128, x_type=f), x, torch.empty(4, 128, device="cuda"), e8(1 << 20))    # fp32 results
    assert mx.last_device_status() == mx.OK
