"""The microscaled operators together, as a training step of a gated feed-forward block uses them: products in 4 bits forward and for the
inputs' gradients, inputs kept in 8 bits, weight gradients from those; eagerly, captured and replayed, and on two streams at once."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

FMT = ref.MXFP4


def new4(rows, cols):
    return (torch.empty((rows, ref.up(cols, 32) // 2), dtype=torch.uint8, device="cuda"),
            torch.empty(sparq.sparq_mx_scale_bytes(FMT, rows, cols), dtype=torch.uint8, device="cuda"))


def new8(rows, cols):
    return (torch.empty((rows, ref.up(cols, 32)), dtype=torch.int8, device="cuda"),
            torch.empty((rows, ref.up(ref.up(cols, 32) // 32, 16)), dtype=torch.uint8, device="cuda"))


def quant(x):
    t = new4(*x.shape)
    sparq.sparq_quantize_mx(x, FMT, *t)
    return t


class Block:
    """y = W2 (silu(W1 x) * (V1 x)); W1 and V1 are the halves of one matrix."""

    def __init__(self, seed, tokens, d, hidden):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        bf = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x, self.dy = rnd(tokens, d).bfloat16(), bf(tokens, ref.up(d, 8))[:, :d]         # rows of 16-byte pieces
        self.dy.copy_(rnd(tokens, d) * 1e-2)
        self.w1, self.w2 = rnd(2 * hidden, d) * d ** -0.5, rnd(d, hidden) * hidden ** -0.5
        self.q = [quant(w) for w in (self.w1, self.w2, self.w1.T.contiguous(), self.w2.T.contiguous())]
        self.h, self.a, self.y, self.dh, self.da, self.dx = bf(tokens, 2 * hidden), bf(tokens, hidden), bf(tokens, d), bf(tokens, 2 * hidden), bf(tokens, hidden), bf(tokens, d)
        self.dw1, self.dw2 = torch.zeros((2 * hidden, d), device="cuda"), torch.zeros((d, hidden), device="cuda")
        self.t = [new4(tokens, d), new4(tokens, hidden), new4(tokens, d), new4(tokens, 2 * hidden)]
        self.kx, self.kg, self.ku, self.ka = new8(tokens, d), new8(tokens, hidden), new8(tokens, hidden), new8(tokens, hidden)
        self.hidden = hidden

    def step(self):
        n = self.hidden
        gate, up = self.h[:, :n], self.h[:, n:]
        # forward
        sparq.sparq_quantize_mx(self.x, FMT, *self.t[0])
        sparq.sparq_quantize_mx(self.x, sparq.FORMAT_MXINT8, *self.kx)
        sparq.sparq_gemm_mxf4(*self.t[0], *self.q[0], FMT, bf16_out=self.h)
        sparq.sparq_act_forward_mx8(gate, sparq.ACT_SILU, self.a, *self.kg, up=up, up_codes=self.ku[0], up_scales=self.ku[1])
        sparq.sparq_quantize_mx(self.a, FMT, *self.t[1])
        sparq.sparq_quantize_mx(self.a, sparq.FORMAT_MXINT8, *self.ka)
        sparq.sparq_gemm_mxf4(*self.t[1], *self.q[1], FMT, bf16_out=self.y)
        # backward
        sparq.sparq_wgrad_mx8(self.dy, *self.ka, self.dw2, accumulate=True)
        sparq.sparq_quantize_mx(self.dy, FMT, *self.t[2])
        sparq.sparq_gemm_mxf4(*self.t[2], *self.q[3], FMT, bf16_out=self.da)
        sparq.sparq_act_backward_mx8(self.da, *self.kg, sparq.ACT_SILU, self.dh[:, :n], up_codes=self.ku[0], up_scales=self.ku[1], dup=self.dh[:, n:])
        sparq.sparq_wgrad_mx8(self.dh, *self.kx, self.dw1, accumulate=True)
        sparq.sparq_quantize_mx(self.dh, FMT, *self.t[3])
        sparq.sparq_gemm_mxf4(*self.t[3], *self.q[2], FMT, bf16_out=self.dx)

    def results(self):
        return [t.clone() for t in (self.y, self.dx, self.dw1, self.dw2)]


def f64(t):
    return t.double().cpu().numpy()


def close(got, want, size, rel):
    far = np.abs(f64(got) - want) - rel * size
    assert far.max() <= 0, far.max()


@pytest.mark.parametrize("tokens,d,hidden", [(1, 64, 96), (37, 100, 72), (200, 256, 320)])
def test_a_step_against_64_bits(tokens, d, hidden):
    """Each operator's output from the outputs that its inputs came from, so that every stage is held to its own rounding."""
    b = Block(tokens, tokens, d, hidden)
    b.step()
    sparq.sparq_check()
    thru = lambda t, fmt=FMT: ref.values(*ref.quantize(t.float().cpu().numpy(), fmt), fmt, t.shape[1])  # noqa: E731
    half, acc = 2.0 ** -8, (hidden * 2 + d + 4608) / 64 * 2.0 ** -23
    n = hidden
    # forward products: half a step of bf16 and the sums' rounding (see test_gpu_mx_gemm.py)
    for a, w, out in ((b.x, b.w1, b.h), (b.a, b.w2, b.y), (b.dy, b.w2.T, b.da), (b.dh, b.w1.T, b.dx)):
        va, vw = thru(a), thru(w.contiguous())
        close(out, va @ vw.T, half * np.abs(va @ vw.T) + 2 * acc * (np.abs(va) @ np.abs(vw).T), 1.0)
    # the block's own function: half a step, and a few units of fp32
    g, u = f64(b.h[:, :n]), f64(b.h[:, n:])
    s = 1 / (1 + np.exp(-g))
    close(b.a, g * s * u, np.abs(g * s * u), half + 40 * 2.0 ** -23)
    g, u, da = thru(b.h[:, :n], ref.MXINT8), thru(b.h[:, n:], ref.MXINT8), f64(b.da)
    s = 1 / (1 + np.exp(-g))
    close(b.dh[:, n:], da * g * s, np.abs(da * g * s), half + 40 * 2.0 ** -23)
    close(b.dh[:, :n], da * u * (s + g * s * (1 - s)), half * np.abs(da * u * (s + g * s * (1 - s))) + 60 * 2.0 ** -23 * np.abs(da * u) * (1 + np.abs(g)), 1.0)
    # weight gradients (see test_gpu_mx_wgrad.py)
    for dy, x, dw in ((b.dy, b.a, b.dw2), (b.dh, b.x, b.dw1)):
        v, dy = thru(x, ref.MXINT8), f64(dy)
        close(dw, dy.T @ v, np.abs(dy).T @ np.abs(v), (57 + tokens / 512) * 2.0 ** -23)


def test_captured_and_replayed():
    eager, graphed = Block(3, 300, 256, 384), Block(3, 300, 256, 384)
    graphed.step()                     # kernels loaded before the capture
    graphed.dw1.zero_()
    graphed.dw2.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for i in range(3):
        for b in (eager, graphed):
            b.x.copy_(torch.randn(b.x.shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(eager.results(), graphed.results()):
            assert torch.equal(a, c)


def test_two_streams_at_once():
    blocks = [Block(i, 500, 512, 768) for i in range(2)]
    want = []
    for b in blocks:
        b.step()
        b.step()
        torch.cuda.synchronize()
        want.append(b.results())
    again = [Block(i, 500, 512, 768) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in again]
    for _ in range(2):
        for b, st in zip(again, streams):
            with torch.cuda.stream(st):
                b.step()
    torch.cuda.synchronize()
    sparq.sparq_check()
    for b, w in zip(again, want):
        for a, c in zip(b.results(), w):
            assert torch.equal(a, c)


def test_decoding_one_token_at_a_time():
    """A token by itself gives the bits that it gives among others, through the block's products."""
    b = Block(5, 16, 256, 320)
    b.step()
    one = Block(5, 1, 256, 320)
    one.q = b.q
    for i in (0, 7, 15):
        one.x.copy_(b.x[i:i + 1])
        one.step()
        assert torch.equal(one.h, b.h[i:i + 1]) and torch.equal(one.a, b.a[i:i + 1])


def test_stream_argument():
    x = torch.randn((40, 64), device="cuda")
    st = torch.cuda.Stream()
    want, t = quant(x), new4(40, 64)
    torch.cuda.synchronize()
    sparq.sparq_quantize_mx(x, FMT, *t, stream=st)
    st.synchronize()
    assert torch.equal(t[0], want[0]) and torch.equal(t[1], want[1])
