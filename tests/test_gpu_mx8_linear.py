"""The product on 8-bit floats with bias, activation and residual in its epilogue against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx8_oracle as mx
from paper_2602_21140_amd import binding, mx8_linear, mx8_pack, mx8_quantize
from test_gpu_mx8 import sum_error

pytestmark = pytest.mark.gpu

class Product:
    def __init__(self, rows, K, N, seed=0):
        rng = np.random.default_rng(seed + rows + K + N)
        x, w = rng.standard_normal((rows, K)) * np.exp(rng.standard_normal((rows, 1))), rng.standard_normal((N, K)) * K ** -0.5
        self.N = N
        self.form = mx8_quantize(torch.from_numpy(x).float().cuda())
        w_form = mx8_quantize(torch.from_numpy(w).float().cuda())
        self.w = mx8_pack(*w_form)
        self.bias = torch.from_numpy(rng.standard_normal(N)).float().cuda()
        self.residual = torch.from_numpy(3 * rng.standard_normal((rows, N))).to(torch.bfloat16).cuda()
        self.x64, self.w64 = (mx.values(*(t.cpu().numpy() for t in form)) for form in (self.form, w_form))

    def run(self, bias=True, activation="none", residual=True, **kw):
        return mx8_linear(*self.form, self.w, self.N, bias=self.bias if bias else None, activation=activation,
                          residual=self.residual if residual else None, **kw)

    def check(self, out, bias=True, activation="none", residual=True):
        """The sum's error, through an activation whose slope is below 1.13 and which is itself exact to 8 roundings, two more additions,
        and the rounding of the result (2^-8).  All elements together, whose errors are independent: the rounding is evenly spread, 2^-8 /
        sqrt(3) of them, beside which the sums' 2^-12 at most is little."""
        z, error = self.x64 @ self.w64.T, sum_error(self.x64, self.w64.T)
        if bias:
            z = z + f64(self.bias)
            error = error + 2.0 ** -24 * np.abs(z)
        want = mx.activated(z, activation)
        error = 1.13 * error + 2.0 ** -21 * np.abs(want)
        if activation == "gelu":  # beside its zero the function's factor is as exact as its argument
            error = error + 2.0 ** -21 * np.abs(z) * np.minimum(1, np.exp(-z * z / 2) * (1 + z * z))
        if residual:
            want = want + f64(self.residual)
            error = error + 2.0 ** -24 * np.abs(want)
        allowed = error * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want) + 1e-38
        off = np.abs(f64(out) - want)
        assert out.dtype is torch.bfloat16 and (off <= allowed).all(), (float((off / allowed).max()), np.argwhere(~(off <= allowed))[:4].tolist())
        assert off.size < 1000 or np.linalg.norm(off) <= 2.0 ** -8 * np.linalg.norm(want)


# a row and a few, every number of 16-row blocks of a tile and one more, several tiles, a large tile and beside it; K below a step,
# with a rest, with fewer steps than wavefronts share; columns that end anywhere in a set of 8, 32, 64, a panel
SIZES = [(1, 32, 1), (1, 128, 7), (2, 96, 33), (1, 4096, 512), (3, 1056, 129), (16, 1024, 64), (17, 160, 65), (32, 512, 100), (33, 2080, 257), (48, 288, 31),
         (64, 640, 300), (65, 32, 24), (200, 1184, 8), (255, 256, 640), (256, 128, 256), (300, 2208, 511), (513, 96, 1000), (1030, 800, 264)]


@pytest.mark.parametrize("rows,K,N", SIZES)
def test_linear(rows, K, N):
    p = Product(rows, K, N)
    p.check(p.run())
    p.check(p.run(bias=False, residual=False), bias=False, residual=False)


@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows", [5, 70, 400])
def test_epilogues(rows, activation):
    p = Product(rows, 224, 77, seed=1)
    for bias in (True, False):
        for residual in (True, False):
            how = dict(bias=bias, activation=activation, residual=residual)
            p.check(p.run(**how), **how)


@pytest.mark.parametrize("rows", [1, 16, 20, 64, 300])
def test_strided_unaligned_and_in_place(rows):
    p = Product(rows, 416, 203, seed=2)
    want = p.run()
    wide = torch.full((2, rows, 260), 7.0, dtype=torch.bfloat16, device="cuda")
    out, res = wide[0, :, 5:208], wide[1, :, 3:206]
    res.copy_(p.residual)
    p.residual = res
    assert torch.equal(p.run(out=out), want)
    out.fill_(7.0)
    assert bool((wide[0] == 7.0).all())  # nothing beside the rows was written
    p.run(out=res)
    assert torch.equal(res, want)
    # codes and scales that begin anywhere they may, weights at 16 bytes
    flat = [torch.zeros(t.numel() + n, dtype=torch.uint8, device="cuda")[n:] for t, n in zip(p.form, (16, 1))]
    for to, t in zip(flat, p.form):
        to.copy_(t.flatten())
    p.form = tuple(to.view(t.shape) for to, t in zip(flat, p.form))
    p.residual = res.copy_(torch.zeros_like(res))
    first = p.run(out=out)
    p.check(first)


@pytest.mark.parametrize("rows", [1, 7, 40, 300])
def test_rows_that_are_not_finite_stay_alone(rows):
    p = Product(rows, 288, 150, seed=3)
    clean = p.run()
    bad = rows // 2
    p.form[1][bad, 4] = 255  # a block that is not finite
    p.form[0][0, 287] = 0x7F if rows > 1 else p.form[0][0, 287]  # a single NaN in the last block
    out = p.run(activation="none")
    others = [r for r in range(rows) if r not in (bad, 0)]
    assert bool(out[bad].isnan().all()) and torch.equal(out[others], clean[others]) and (rows == 1 or bool(out[0].isnan().all()))
    assert bool(p.run(activation="relu", residual=False)[bad].isnan().all())


def test_what_lies_behind_a_row_is_not_read():
    """Bytes of NaN behind the last row and beyond K's end of the others."""
    for rows in (3, 40, 300):
        for K in (32, 96, 160, 224):
            p = Product(rows, K, 70, seed=4)
            want = p.run()
            n = K // 32
            codes = torch.full((rows * K + 256,), 0x7F, dtype=torch.uint8, device="cuda")
            scales = torch.full((rows * n + 256,), 255, dtype=torch.uint8, device="cuda")
            codes[:rows * K], scales[:rows * n] = p.form[0].flatten(), p.form[1].flatten()
            p.form = codes[:rows * K].view(rows, K), scales[:rows * n].view(rows, n)
            assert torch.equal(p.run(), want)


@pytest.mark.parametrize("rows", [9, 300])
def test_streams_graphs_and_no_rows(rows):
    p = Product(rows, 512, 320, seed=5)
    want = p.run()
    assert mx8_linear(p.form[0][:0], p.form[1][:0], p.w, p.N).shape == (0, 320)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = p.run(stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        p.run(out=out)
    for i in range(4):
        mx8_quantize(torch.randn(rows, 512, generator=torch.Generator().manual_seed(i)).cuda(), out=p.form)
        want = p.run()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_library_refuses():
    p = Product(4, 64, 40)
    L, x, s, w = binding.lib(), p.form[0].data_ptr(), p.form[1].data_ptr(), p.w.data_ptr()
    out, b = p.residual.data_ptr(), p.bias.data_ptr()
    good = [x, s, 0, 64, w, 40, b, 0, out, 40, out, 40, None]
    assert L.revive_mx_eight_linear(*good) == 0
    good[2] = 4
    for i, v in ((0, 0), (1, 0), (2, -1), (3, 0), (3, 63), (4, 0), (5, 0), (5, 1 << 27), (7, 4), (7, -1), (9, 39), (9, 41), (10, 0), (11, 39),
                 (0, x + 8), (4, w + 8), (6, b + 2), (8, out + 1), (10, out + 1)):
        bad = list(good)
        bad[i] = v
        assert L.revive_mx_eight_linear(*bad) == -1 and L.revive_last_error(None), (i, v)
    torch.cuda.synchronize()
