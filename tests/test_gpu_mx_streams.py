"""The calls on microscaled matrices and the norm as a training step makes them, one after the other: on a stream of their own, captured in a
graph, through either call path, and against 64 bits from end to end."""
import itertools

import mx_reference as R
import numpy as np
import pytest
import torch
from test_gpu_mx import DEV, matrix, operand

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5


class Layer:
    """h = x + residual; y = norm(h) in 8 bits; out = y w^T with w in 4 bits; and back: dy from dout and w, the weight's gradient and the norm's
    into fp32 rows that hold something already."""

    def __init__(self, tokens, width, out, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=gen).to(DEV)   # noqa: E731
        self.x, self.residual, self.dout = r(tokens, width).to(dtype), r(tokens, width).to(dtype), r(tokens, out).to(dtype)
        self.gain, self.w = 1 + 0.1 * r(width), 0.05 * r(out, width)
        self.noise = torch.randint(256, (tokens, out), dtype=torch.uint8, generator=gen).to(DEV)
        E2, E4 = B.NT_MX_E2M1, B.NT_MX_E4M3
        self.w_mx, self.w_t = B.make_mx(out, width, E2, DEV), B.make_mx(width, out, E2, DEV)
        self.y_mx, self.y_t = B.make_mx(tokens, width, E4, DEV), B.make_mx(width, tokens, E4, DEV)
        self.d_mx, self.d_t = B.make_mx(tokens, out, E4, DEV), B.make_mx(out, tokens, E4, DEV)
        self.h, self.y, self.dy, self.dx = (torch.empty_like(self.x) for _ in range(4))
        self.rstd, self.out = torch.empty(tokens, device=DEV), torch.empty(tokens, out, dtype=dtype, device=DEV)
        self.row = r(width * out + width + 3)          # a row of the norm test: the weight's gradient begins at an odd element
        self.dw, self.dgain = self.row[1:1 + out * width].view(out, width), self.row[1 + out * width:1 + out * width + width]
        need = lambda a, b, t: B.normtest_mx_matmul_workspace_bytes(a, b, t)   # noqa: E731
        size = max(need(self.y_mx, self.w_mx, dtype), need(self.d_mx, self.w_t, dtype), need(self.d_t, self.y_t, torch.float32),
                   B.normtest_rms_norm_workspace_bytes(tokens, width), 16)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=DEV)

    def step(self, stream=None):
        k = dict(stream=stream)
        B.normtest_mx_quantize(self.w, self.w_mx, self.w_t, **k)
        B.normtest_rms_norm(self.x, self.gain, self.y, residual=self.residual, eps=EPS, sum_out=self.h, out_mx=self.y_mx, rstd=self.rstd, **k)
        B.normtest_mx_matmul(self.y_mx, self.w_mx, self.out, workspace=self.workspace, **k)
        B.normtest_mx_quantize(self.dout, self.d_mx, self.d_t, fit=True, noise=self.noise, **k)
        B.normtest_mx_quantize(self.y, None, self.y_t, **k)
        B.normtest_mx_matmul(self.d_mx, self.w_t, self.dy, workspace=self.workspace, **k)
        B.normtest_mx_matmul(self.d_t, self.y_t, self.dw, scale=0.5, beta=1.0, workspace=self.workspace, **k)
        B.normtest_rms_norm_backward(self.dy, self.h, self.gain, self.rstd, self.dx, dsum=self.residual, dweight=self.dgain, scale=0.5, beta=1.0,
                                     workspace=self.workspace, **k)

    def results(self):
        return [t.clone() for t in (self.w_mx.codes, self.w_t.codes, self.y_mx.codes, self.y_mx.scales, self.h, self.y, self.rstd, self.out, self.d_mx.codes,
                                    self.d_t.codes, self.dy, self.dx, self.row)]


SIZES = [(1, 96, 40), (70, 200, 333), (300, 1024, 512)]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_layer_against_64_bits(sizes):
    """Every product from what the step before left, which the tests of each call cover; here that they fit together."""
    s = Layer(*sizes)
    before = R.wide(s.row)
    s.step()
    near = lambda got, want, rel: np.linalg.norm(R.wide(got) - want) <= rel * np.linalg.norm(want)   # noqa: E731
    w, w_t, y, y_t, d, d_t = (R.numbers(m) for m in (s.w_mx, s.w_t, s.y_mx, s.y_t, s.d_mx, s.d_t))
    assert np.array_equal(w, R.quantized(R.wide(s.w), B.NT_MX_E2M1)) and np.array_equal(w_t, R.quantized(R.wide(s.w).T, B.NT_MX_E2M1))
    assert np.array_equal(d_t, R.quantized(R.wide(s.dout).T, B.NT_MX_E4M3, True, s.noise.cpu().numpy().T))
    assert np.array_equal(y_t, R.quantized(R.wide(s.y).T, B.NT_MX_E4M3))
    # in bf16, half a step of 2^-8 at most, and 8-bit products' 4e-5
    assert near(s.out, y @ w.T, 2.0 ** -9 + 1e-4) and near(s.dy, d @ w_t.T, 2.0 ** -9 + 1e-4)
    tokens, width, out = sizes
    dw = before[1:1 + out * width].reshape(out, width) + 0.5 * d_t @ y_t.T
    assert near(s.dw, dw, 1e-6)
    hat = R.wide(s.h) * R.wide(s.rstd)[:, None]
    g = R.wide(s.dy) * R.wide(s.gain)
    dx = R.wide(s.rstd)[:, None] * (g - hat * (g * hat).mean(1, keepdims=True)) + R.wide(s.residual)
    assert near(s.dx, dx, 2.0 ** -9 + 1e-5)
    assert near(s.dgain, before[1 + out * width:1 + out * width + width] + 0.5 * (R.wide(s.dy) * hat).sum(0), 1e-6)
    assert np.array_equal(R.wide(s.row)[[0, -2, -1]], before[[0, -2, -1]])


@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_graph(sizes):
    """Captured and replayed, with other work between: every replay gives the eager bits; what accumulates goes on accumulating."""
    s, eager = Layer(*sizes), Layer(*sizes)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    eager.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for k in range(4):
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for a, b in zip(s.results(), eager.results()):
            assert torch.equal(a, b)
        for t in (s.x, eager.x):
            t.mul_(0.5 + 0.25 * k)
        _ = (torch.randn(1 << 16, device=DEV) * 2).sum().item()


def test_two_graphs_with_a_workspace_each():
    """Two layers, each captured with memory of its own, replayed in turn and on two streams at once."""
    layers, wants, graphs = [Layer(64, 512, 96, seed=k) for k in range(2)], [], []
    for k in range(2):
        e = Layer(64, 512, 96, seed=k)
        for _ in range(3):
            e.step()
        wants.append(e.results())
    for s in layers:
        s.step()      # warm
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for st, g in zip(streams, graphs):
        with torch.cuda.stream(st):
            g.replay()
    torch.cuda.synchronize()
    for s, want in zip(layers, wants):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), want))


def test_other_stream():
    """On a stream given by the caller, with workspaces and results made by the calls."""
    want, s = Layer(40, 3000, 70), Layer(40, 3000, 70)
    want.step()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    s.workspace = None
    s.step(stream=st)
    out = B.normtest_mx_matmul(s.y_mx, s.w_mx, dtype=torch.float32, stream=st)
    values = B.normtest_mx_dequantize(s.y_mx, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.results(), want.results()))
    assert torch.equal(out, B.normtest_mx_matmul(s.y_mx, s.w_mx, dtype=torch.float32)) and torch.equal(values, B.normtest_mx_dequantize(s.y_mx))


def test_paths_agree(monkeypatch):
    """The native call path and the checks in Python give the same bits, with and without workspaces, and the same refusals."""
    a, b = Layer(50, 700, 90), Layer(50, 700, 90)
    assert B._fast is not None and a.w_mx.native
    a.step()
    b.workspace = None
    b.step()
    assert all(torch.equal(x, y) for x, y in zip(a.results(), b.results()))
    c = Layer(50, 700, 90)
    with monkeypatch.context() as m:
        m.setattr(B, "_fast", None)
        c.step()
    assert all(torch.equal(x, y) for x, y in zip(a.results(), c.results()))

    def refusals():
        bad = [lambda: B.normtest_mx_matmul(a.y_mx, a.w_t, a.out), lambda: B.normtest_mx_matmul(a.y_mx, a.w_mx, a.out.t()),
               lambda: B.normtest_mx_matmul(a.y_mx, a.w_mx, a.out, scale=float("nan")), lambda: B.normtest_mx_matmul(a.y_mx, a.w_mx, a.out.cpu()),
               lambda: B.normtest_mx_matmul(a.y_mx, a.w_mx, beta=1.0), lambda: B.normtest_mx_quantize(a.x, a.w_mx),
               lambda: B.normtest_mx_quantize(a.x, None, None), lambda: B.normtest_mx_quantize(a.x, a.y_mx, noise=a.noise),
               lambda: B.normtest_mx_dequantize(a.y_mx, a.out), lambda: B.normtest_rms_norm(a.x, a.gain[:-1], a.y),
               lambda: B.normtest_rms_norm(a.x, a.gain, a.y.float()), lambda: B.normtest_rms_norm(a.x, a.gain, a.y, eps=0.0),
               lambda: B.normtest_rms_norm(a.x, a.gain, out_mx=a.w_mx), lambda: B.normtest_rms_norm_backward(a.dy, a.h, a.gain, a.rstd[:-1], a.dx),
               lambda: B.normtest_rms_norm_backward(a.dy, a.h, a.gain, a.rstd), lambda: B.normtest_rms_norm_backward(a.dy, a.h[:-1], a.gain, a.rstd, a.dx),
               lambda: B.normtest_rms_norm_backward(a.dy, a.h, a.gain, a.rstd, a.dx, dweight=a.dgain, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))]
        seen = []
        for call in bad:
            with pytest.raises((ValueError, TypeError, RuntimeError)) as e:
                call()
            seen.append((type(e.value), str(e.value)))
        return seen
    native = refusals()
    with monkeypatch.context() as m:
        m.setattr(B, "_fast", None)
        assert refusals() == native
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.results(), c.results()))     # nothing was written


def test_moved_matrix_is_noticed():
    m = operand(4, 64, "e2m1", 0)
    m.codes.data = torch.zeros_like(m.codes)
    with pytest.raises(RuntimeError, match="other memory"):
        B.normtest_mx_dequantize(m, torch.empty(4, 64, device=DEV))


def test_columns_of_one_matrix():
    """Slices of rows and of whole blocks of a microscaled matrix are matrices; what lies beside them is not touched."""
    x = matrix(64, 256, torch.bfloat16, 3)
    whole = B.make_mx(64, 256, B.NT_MX_E4M3, DEV)
    whole.codes.fill_(0x11)
    part = B.MxTensor(whole.codes[16:48, 64:192], whole.scales[16:48, 2:6], 128, B.NT_MX_E4M3)
    B.normtest_mx_quantize(x[16:48, 64:192], part)
    assert np.array_equal(R.numbers(part), R.quantized(R.wide(x[16:48, 64:192]), B.NT_MX_E4M3))
    rest = whole.codes.clone()
    rest[16:48, 64:192] = 0x11
    assert (rest == 0x11).all()
    b = operand(20, 128, "e2m1", 1)
    got = B.normtest_mx_matmul(part, b, dtype=torch.float32)
    want = R.numbers(part) @ R.numbers(b).T
    assert np.linalg.norm(R.wide(got) - want) <= 1e-6 * np.linalg.norm(np.abs(R.numbers(part)) @ np.abs(R.numbers(b)).T)


def test_far_offsets():
    """Rows so far apart that byte offsets pass 32 bits: the product of few rows serves them, of more rows too."""
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB")
    ld = 1 << 26
    memory = torch.zeros(80 * ld, dtype=torch.uint8, device=DEV)
    codes = memory.view(80, ld)[:, :512]
    scales = memory.view(80, ld)[:, 4096:4096 + 32]
    a, b = B.MxTensor(codes, scales, 1024, B.NT_MX_E2M1), operand(33, 1024, "e2m1", 2)
    x = matrix(80, 1024, torch.float32, 4)
    B.normtest_mx_quantize(x, a)
    assert np.array_equal(R.numbers(a), R.quantized(R.wide(x), B.NT_MX_E2M1))
    for rows, cols in ((a, b), (b, a)):
        got = B.normtest_mx_matmul(rows, cols, dtype=torch.float32)
        na, nb = R.numbers(rows), R.numbers(cols)
        assert np.linalg.norm(R.wide(got) - na @ nb.T) <= 1e-6 * np.linalg.norm(np.abs(na) @ np.abs(nb).T)


@pytest.mark.parametrize("fa,fb", itertools.product(("e2m1", "e4m3"), repeat=2))
def test_scales_at_any_address(fa, fb):
    """Scales that begin at an odd byte, in rows of an odd length."""
    a, b = operand(70, 1100, fa, 1), operand(130, 1100, fb, 2)
    memory = torch.full((130 * 37 + 8,), 255, dtype=torch.uint8, device=DEV)
    odd = memory[1:1 + 130 * 37].view(130, 37)[:, :35]
    odd.copy_(b.scales[:, :35])
    c = B.MxTensor(b.codes, odd, 1100, b.format)
    for dtype in (torch.bfloat16, torch.float32):
        assert torch.equal(B.normtest_mx_matmul(a, c, dtype=dtype), B.normtest_mx_matmul(a, b, dtype=dtype))
        assert torch.equal(B.normtest_mx_matmul(c, a, dtype=dtype), B.normtest_mx_matmul(b, a, dtype=dtype))
