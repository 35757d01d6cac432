"""The residual norm with its 8-bit output against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx8_oracle as mx
from paper_2602_21140_amd import add_rms_norm, binding

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def draw(rows, H, dtype, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, H)) * np.exp(rng.standard_normal((rows, 1)))
    r = 3 * rng.standard_normal((rows, H))
    if rows > 2:
        x[1], r[1] = 0, 0
    return [torch.from_numpy(v).to(dtype).cuda() for v in (x, r, 1 + 0.3 * rng.standard_normal(H))]


def check(x, residual, weight, eps, total, y, codes, scales):
    """The stored sum bit by bit; y within three roundings of fp32 (the root's reciprocal and two products) and its own; the 8-bit
    form that of the stored y, byte by byte."""
    dtype, s = x.dtype, x
    if residual is not None:
        s = (x.float() + residual.float()).to(dtype)  # one sum in fp32, one rounding
        if total is not None:
            assert torch.equal(total, s)
    if y is not None:
        want = mx.rms_norm(f64(s), f64(weight), float(np.float32(eps)))
        # below fp32's normal numbers a rounding is half of 2^-149, or of bf16's 2^-133
        allowed = (3 * 2.0 ** -24 + HALF_STEP[dtype]) * 1.01 * np.abs(want) + (2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -147)
        off = np.abs(f64(y) - want)
        assert (off <= allowed).all(), float((off / allowed).max())
        if codes is not None:
            want_codes, want_scales = mx.quantize(f64(y))
            assert np.array_equal(scales.cpu().numpy(), want_scales) and np.array_equal(codes.cpu().numpy(), want_codes)


# every shape of the kernel: a wavefront a row, 256 threads with one, two and four units, 1024 with two, and rows that are read twice;
# at their borders, odd lengths among them
SIZES = [(1, 1), (5, 7), (3, 32), (9, 512), (4, 513), (2, 2048), (3, 2056), (7, 4095), (2, 4104), (3, 7168), (2, 8192), (3, 8193),
         (2, 16384), (2, 16390), (3, 40000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,H", SIZES)
def test_norm(rows, H, dtype):
    x, r, w = draw(rows, H, dtype, rows + H)
    check(x, r, w, 1e-6, *add_rms_norm(x, w, residual=r, quantize=True))
    check(x, None, w, 1e-5, *add_rms_norm(x, w, eps=1e-5, quantize=True))
    check(x, r, w, 0.5, *add_rms_norm(x, w, residual=r, eps=0.5))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [200, 3500, 12000, 20000])
def test_in_place_strided_unaligned_and_partial_outputs(H, dtype):
    rows = 6
    x, r, w = draw(rows, H, dtype, H)
    total, y, codes, scales = add_rms_norm(x, w, residual=r, quantize=True)
    check(x, r, w, 1e-6, total, y, codes, scales)
    same = lambda got, want: all(torch.equal(a, b) for a, b in zip(got, want))  # noqa: E731
    # the residual stream in place, x in place, both swapped
    for s_to, y_to in ((1, 0), (0, 1), (1, None), (0, None), (None, 0), (None, 1)):
        a, b = x.clone(), r.clone()
        pick = {None: None, 0: a, 1: b}
        s_out = pick[s_to] if s_to is not None else torch.empty_like(x)
        y_out = pick[y_to] if y_to is not None else torch.empty_like(x)
        got = add_rms_norm(a, w, residual=b, quantize=True, out=(s_out, y_out, torch.empty_like(codes), torch.empty_like(scales)))
        assert same(got, (total, y, codes, scales)), (s_to, y_to)
    a = x.clone()
    alone = add_rms_norm(x, w)[1]
    add_rms_norm(a, w, out=(None, a, None, None))
    assert torch.equal(a, alone)
    # without the sum or y; without either
    for keep in ((False, True), (True, False), (False, False)):
        got = add_rms_norm(x, w, residual=r, quantize=True, out=(torch.empty_like(x) if keep[0] else None, torch.empty_like(x) if keep[1] else None,
                                                                  torch.empty_like(codes), torch.empty_like(scales)))
        for g, want in zip(got, (total, y, codes, scales)):
            assert g is None or torch.equal(g, want)
    # rows at odd places of wider ones
    wide = torch.zeros(2, rows, H + 13, dtype=dtype, device="cuda")
    wide[0, :, 3:3 + H], wide[1, :, 5:5 + H] = x, r
    assert same(add_rms_norm(wide[0, :, 3:3 + H], w, residual=wide[1, :, 5:5 + H], quantize=True), (total, y, codes, scales))
    assert torch.equal(add_rms_norm(x[::2], w)[1], alone[::2])
    flat = torch.zeros(2 * (rows * H + 3) + H, dtype=dtype, device="cuda")
    s_out, y_out = flat[1:1 + rows * H].view(rows, H), flat[rows * H + 3:2 * rows * H + 3].view(rows, H)
    assert same(add_rms_norm(x, w, residual=r, out=(s_out, y_out, None, None))[:2], (total, y))
    assert not flat[0] and not flat[1 + rows * H:3 + rows * H].any() and not flat[2 * rows * H + 3:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_any_size(dtype):
    """Squares that fp32 cannot hold, at both ends, with an eps of nothing."""
    x, _, w = draw(12, 640, dtype, 5)
    x[1] = 1.0
    for i, e in enumerate((-125, -100, -70, -40, 40, 64, 100, 120)):
        x[i + 2] = (torch.sign(x[i + 2].float()) * x[i + 2].float().abs().clamp(0.01, 8) * 2.0 ** e).to(dtype)
    check(x, None, w, 0.0, *add_rms_norm(x, w, eps=0.0, quantize=True))
    x.zero_()
    assert bool(add_rms_norm(x, w, eps=0.0)[1].isnan().all()) and not add_rms_norm(x, w)[1].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_are_not_finite_stay_alone(dtype):
    x, r, w = draw(6, 3000, dtype, 6)
    clean = add_rms_norm(x, w, residual=r, quantize=True)
    x[2, 77], r[4, 2999] = float("nan"), float("inf")
    got = add_rms_norm(x, w, residual=r, quantize=True)
    others = [0, 1, 3, 5]
    assert all(torch.equal(g[others], c[others]) for g, c in zip(got, clean))
    assert bool(got[1][2].isnan().all()) and bool((got[3][2] == 255).all())
    # an infinity makes the row's mean infinite: NaN where it is, zeros elsewhere
    assert bool(got[1][4, 2999].isnan()) and not got[1][4, :2999].any() and int(got[3][4, -1]) == 255 and not got[3][4, :-1].any()
    assert bool((got[2][2] == 0x7F).all())


def test_no_rows_other_streams_and_graphs():
    x, r, w = draw(40, 1000, torch.bfloat16, 7)
    assert add_rms_norm(x[:0], w, residual=r[:0], quantize=True)[2].shape == (0, 1024)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = add_rms_norm(x, w, residual=r, quantize=True, stream=s)
    s.synchronize()
    check(x, r, w, 1e-6, *out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        add_rms_norm(x, w, residual=r, quantize=True, out=out)
    for i in range(4):
        x.copy_(draw(40, 1000, torch.bfloat16, 8 + i)[0])
        want = add_rms_norm(x, w, residual=r, quantize=True)
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_rows_beyond_32_bits():
    """The last of so many rows that their elements' numbers pass 2^32."""
    rows, H = (1 << 32) // 4096 + 3, 4096
    x = torch.zeros(rows, H, dtype=torch.bfloat16, device="cuda")
    x[-2:] = draw(2, H, torch.bfloat16, 9)[0]
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    _, y, codes, scales = add_rms_norm(x, w, quantize=True)
    check(x[-3:], None, w, 1e-6, None, y[-3:], codes[-3:], scales[-3:])
    assert not y[:-2].any()


def test_library_refuses():
    x, r, w = draw(4, 64, torch.bfloat16, 0)
    L, p, q, n = binding.lib(), x.data_ptr(), r.data_ptr(), w.data_ptr()
    y = torch.empty(4, 64, dtype=torch.bfloat16, device="cuda").data_ptr()
    codes = torch.empty(4, 64, dtype=torch.uint8, device="cuda").data_ptr()
    good = [p, q, n, 1, 4, 64, 64, 64, 1e-6, q, y, codes, codes, None]
    assert L.revive_add_rms_norm(*[*good[:4], 0, *good[5:]]) == 0
    for i, v in ((0, 0), (2, 0), (3, 2), (4, -1), (5, 0), (5, 1 << 25), (6, 63), (7, 63), (7, 65), (8, -1.0), (8, float("nan")), (8, float("inf")),
                 (12, 0), (11, 0), (11, codes + 8), (0, p + 1), (1, q + 1), (2, n + 1), (9, q + 1), (10, y + 1), (10, q), (1, 0)):
        bad = list(good)
        bad[i] = v
        assert L.revive_add_rms_norm(*bad) == -1 and L.revive_last_error(None), (i, v)
    bad = [*good[:9], 0, 0, 0, 0, None]
    assert L.revive_add_rms_norm(*bad) == -1  # nothing to write
    torch.cuda.synchronize()


# rows that end inside of a unit of eight numbers, with every number of them left over, in the lane that ends a wavefront and in
# the one that begins the next; in place, where the last unit is read beside what another thread writes; more than fits the last-level cache
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [9, 10, 11, 12, 13, 14, 15, 509, 514, 1025, 2839, 6151, 8191, 10003, 16383, 16386, 16391])
def test_rows_that_end_inside_of_a_unit(H, dtype):
    rows = 2100 if H == 2839 else 5  # more rows than workgroups at a time
    x, r, w = draw(rows, H, dtype, H)
    total, y, codes, scales = add_rms_norm(x, w, residual=r, quantize=True)
    check(x, r, w, 1e-6, total, y, codes, scales)
    a, b = x.clone(), r.clone()
    got = add_rms_norm(a, w, residual=b, quantize=True, out=(b, a, torch.empty_like(codes), torch.empty_like(scales)))
    assert all(torch.equal(g, v) for g, v in zip(got, (total, y, codes, scales)))
    guarded = torch.full((2, rows * H + 16), 7.0, dtype=dtype, device="cuda")
    outs = [g[8:8 + rows * H].view(rows, H) for g in guarded]
    add_rms_norm(x, w, residual=r, out=(*outs, None, None))
    assert torch.equal(outs[0], total) and torch.equal(outs[1], y)
    assert bool((guarded[:, :8] == 7.0).all()) and bool((guarded[:, 8 + rows * H:] == 7.0).all())
    x[2, H - 1], r[3, 0] = float("nan"), -float("inf")
    got = add_rms_norm(x, w, residual=r, quantize=True)
    others = [i for i in range(rows) if i not in (2, 3)]
    assert all(torch.equal(g[others], v[others]) for g, v in zip(got, (total, y, codes, scales)))
    assert bool(got[1][2].isnan().all()) and bool((got[3][2] == 255).all()) and bool((got[2][2] == 0x7F).all())
    assert bool(got[1][3, 0].isnan()) and not got[1][3, 1:].any() and int(got[3][3, 0]) == 255 and not got[3][3, 1:].any()


@pytest.mark.parametrize("dtype,H", [(torch.bfloat16, 4099), (torch.float32, 2051), (torch.bfloat16, 4096)])
def test_more_than_the_caches_hold(dtype, H):
    rows = 33000
    x, r, w = draw(64, H, dtype, H)
    many = torch.arange(rows, device="cuda") % 64
    got = add_rms_norm(x[many], w, residual=r[many], quantize=True)
    want = add_rms_norm(x, w, residual=r, quantize=True)
    check(x, r, w, 1e-6, *want)
    assert all(torch.equal(g, v[many]) for g, v in zip(got, want))
