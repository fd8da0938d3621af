"""Root-mean-square norm with the residual's addition, its gradient and its 8-bit
form on the GPU against 64 bits, element by element.

Bounds, with u the roundoff of a stored type and U = 2^-24 of fp32.  A sum over a
row adds at most depth = 80 + cols / 1024 terms one after another (32 in a
thread or cols / 1024 in a wide row's, 5 in a warp, 32 in a block), all of one
sign in the sum of squares: relative error depth U, halved by the root; the mean's
factor, eps, the root and two products are five more roundings."""
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TYPES = [(F32, F32), (BF, F32), (BF, BF)]             # activations, weight
U = 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def make(rows, cols, dtype, weight, seed=0, residual=True):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    channel = torch.exp(randn(cols))
    x = (randn(rows, cols) * channel).to(dtype)
    r = (2 * randn(rows, cols) * channel).to(dtype) if residual else None
    return x, r, (1 + 0.3 * randn(cols)).to(weight), randn(rows, cols).to(dtype), randn(rows, cols).to(dtype)


def depth(cols):
    return 80 + cols / 1024


def forward(x, r, w, eps=EPS):
    """(s as stored, y, r) in 64 bits."""
    s = x if r is None else (x.float() + r.float()).to(x.dtype)
    rstd = (s.double().square().mean(-1) + eps) ** -0.5
    return s, s.double() * rstd[..., None] * w.double(), rstd


def forward_agrees(got, x, r, w, eps=EPS):
    y, s, rstd = got
    S, Y, RS = forward(x, r, w, eps)
    e = (depth(x.shape[-1]) / 2 + 5) * U
    return (torch.equal(s, S) and bool(((rstd.double() - RS).abs() <= e * RS).all())
            and bool(((y.double() - Y).abs() <= (e + R.ROUND[y.dtype]) * Y.abs() + 1e-45).all()))


def gradient_agrees(got, dy, ds, s, w, rstd):
    """The kernel starts from the fp32 rstd that it is given; so does this."""
    dx, dw = got
    cols, rows = s.shape[-1], s.numel() // s.shape[-1]
    S, G, r = s.double(), dy.double() * w.double(), rstd.double()[..., None]
    mean, size = (G * S).mean(-1, keepdim=True), (G * S).abs().mean(-1, keepdim=True)
    want = r * G - S * r ** 3 * mean
    parts = (r * G).abs() + S.abs() * r ** 3 * size
    if ds is not None:
        want, parts = want + ds.double(), parts + ds.double().abs()
    e = (depth(cols) + 10) * U
    ok = ((dx.double() - want).abs() <= e * parts + R.ROUND[dx.dtype] * want.abs() + 1e-45).all()
    terms = (dy.double() * S * r).reshape(-1, cols)
    DW = terms.sum(0)
    # any order of the rows' sum: at most rows - 1 additions, the product with r and dy's
    ok &= ((dw.double() - DW).abs() <= (rows + 3) * U * terms.abs().sum(0) + R.ROUND[dw.dtype] * DW.abs()).all()
    return bool(ok)


SHAPES = [(1, 1), (1, 8), (3, 7), (2, 33), (5, 256), (9, 264), (33, 512), (7, 777), (64, 1024), (3, 1032), (4, 2048), (6, 2055),
          (2, 4096), (3, 16384), (2, 16385), (2, 16392), (2, 32768), (2, 32769), (2, 40000), (700, 128), (3000, 96), (1000, 1536)]


@pytest.mark.parametrize("dtype,weight", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_values_and_gradients(dtype, weight, rows, cols):
    for residual in (True, False):
        x, r, w, dy, ds = make(rows, cols, dtype, weight, residual=residual)
        got = api.rms_norm(x, r, w)
        assert forward_agrees(got, x, r, w)
        _, s, rstd = got
        for h in ((ds, None) if residual else (None,)):
            assert gradient_agrees(api.rms_norm_grad(dy, h, s, w, rstd), dy, h, s, w, rstd)


def eight_agrees(q, scales, Y, cols):
    """Scales are the smallest that fit, values within half a step of y; y itself
    carries the relative error e of its fp32 arithmetic."""
    e = (depth(cols) / 2 + 5) * U
    n = scales.shape[-1]
    pad = torch.nn.functional.pad(Y, (0, 32 * n - cols)).view(-1, n, 32)
    top, k = pad.abs().amax(2), scales.reshape(-1, n).double() - 127
    ok = (top <= 448 * 2.0 ** k * (1 + e)).all() & ((k == -127) | (top > 224 * 2.0 ** k * (1 - e))).all()
    unit = (2.0 ** k).repeat_interleave(32, 1)[:, :cols]
    Y = Y.reshape(-1, cols)
    value = q.float().double().reshape(-1, cols) * unit
    # half a step: 2^-4 of the value, or of the smallest normal number 2^-6
    half = 2.0 ** -4 * torch.maximum(Y.abs(), 2.0 ** -6 * unit)
    return bool(ok) and bool(((value - Y).abs() <= half + 2 * e * Y.abs()).all())


@pytest.mark.parametrize("dtype,weight", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_eight_bits(dtype, weight, rows, cols):
    x, r, w, _, _ = make(rows, cols, dtype, weight, seed=3)
    q, scales, y, s, rstd = api.rms_norm_8bit(x, r, w, with_y=True)
    assert forward_agrees((y, s, rstd), x, r, w)
    assert eight_agrees(q, scales, forward(x, r, w)[1], cols)
    q2, scales2, s2 = api.rms_norm_8bit(x, r, w)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scales2, scales) and torch.equal(s2, s)
    unit = torch.pow(2.0, scales.double() - 127).repeat_interleave(32, 1)[:, :cols]
    for t in (BF, F32):
        assert torch.equal(api.decode_8bit(q, scales, dtype=t), (q.float().double() * unit).to(t))


@pytest.mark.parametrize("dtype,weight", TYPES)
@pytest.mark.parametrize("rows,cols", [(4000, 512), (3000, 777), (1000, 2048), (700, 1536), (100, 20000)])
def test_eight_bits_round_as_64_bits_do(dtype, weight, rows, cols):
    """The sum of squares has at most 11 roundings one after another (10 in a thread of a
    warp's row; 4 and 2 in a thread and 5 in a warp of a block's; one and 5 in a wide
    row's), all of one sign, the rest is exact to less than 2^-24, and y is rounded once:
    y is off by (11 / 2 + 2) 2^-24, and its code is one of those at either end."""
    x, r, w, _, _ = make(rows, cols, dtype, weight, seed=11)
    eps = 2.0 ** -20
    q, scales, _ = api.rms_norm_8bit(x, r, w, eps=eps)
    Y = forward(x, r, w, eps)[1]
    pad = torch.nn.functional.pad(Y, (0, -cols % 32)).view(rows, -1, 32)
    mantissa, k = torch.frexp(pad.abs().amax(2))           # top = mantissa 2^k, mantissa in 0.5 .. 1
    k = (k - 9 + (mantissa > 0.875).int()).clamp(-127, 127)
    assert torch.equal(scales, (k + 127).to(torch.uint8))
    unit = torch.pow(2.0, k.double()).repeat_interleave(32, 1)[:, :cols]
    e = (11 / 2 + 2) * U
    ends = [(Y / unit * (1 + sign * e)).float().to(torch.float8_e4m3fn).float() for sign in (-1, 1)]
    got = q.float()
    assert bool(((got == ends[0]) | (got == ends[1])).all())


def test_eight_bit_limits():
    """Zeros, magnitudes at both ends of the exponents, and groups that hold an
    infinity or NaN."""
    w = torch.ones(96, device="cuda")
    x = torch.zeros(3, 96, device="cuda")
    q, scales, _ = api.rms_norm_8bit(x, None, w)
    assert bool((scales == 0).all()) and bool((api.decode_8bit(q, scales, dtype=F32) == 0).all())
    x = torch.ones(1, 96, device="cuda")
    for size in (1e-38, 1e-30, 448.0, 449.0, 3e38):
        w = torch.full((96,), size, device="cuda")
        w[:32] *= torch.linspace(-1, 1, 32, device="cuda")
        q, scales, _ = api.rms_norm_8bit(x, None, w, eps=0.0)
        assert eight_agrees(q, scales, w.double()[None], 96)
    w = torch.ones(96, device="cuda")
    w[40], w[70] = float("inf"), float("nan")
    q, scales, _ = api.rms_norm_8bit(x, None, w, eps=0.0)
    assert scales.tolist() == [[127 - 8, 255, 255]]
    y = api.decode_8bit(q, scales, dtype=F32)
    assert bool((y[0, :32] == 1).all()) and bool(y[0, 32:].isnan().all())


def test_every_code_decodes():
    q = torch.arange(256, device="cuda", dtype=torch.uint8).repeat(256, 1).view(torch.float8_e4m3fn)
    scales = torch.arange(256, device="cuda", dtype=torch.uint8)[:, None].repeat(1, 8)
    unit = torch.pow(2.0, torch.arange(256, device="cuda", dtype=torch.float64) - 127)
    unit[255] = float("nan")
    want = q.float().double() * unit[:, None]
    for t in (F32, BF):
        got = api.decode_8bit(q, scales, dtype=t)
        assert torch.equal(torch.nan_to_num(got.double(), nan=-7.0, posinf=9e99), torch.nan_to_num(want.to(t).double(), nan=-7.0, posinf=9e99))


def test_rows_without_size_and_not_finite():
    x, r, w, dy, ds = make(6, 40, F32, F32)
    x[0], r[0] = 0.0, 0.0
    x[1, 3], x[2, 5] = float("inf"), float("nan")
    y, s, rstd = api.rms_norm(x, r, w)
    assert bool((y[0] == 0).all()) and abs(float(rstd[0]) - EPS ** -0.5) < 1e-3
    assert float(rstd[1]) == 0 and bool(y[2].isnan().all())
    fine = slice(3, 6)
    assert forward_agrees((y[fine], s[fine], rstd[fine]), x[fine], r[fine], w)
    dx, _ = api.rms_norm_grad(dy, ds, s, w, rstd)
    assert gradient_agrees((dx[fine], api.rms_norm_grad(dy[fine], ds[fine], s[fine], w, rstd[fine])[1]), dy[fine], ds[fine], s[fine], w, rstd[fine])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cols", [40, 45, 512, 2048, 17000])
def test_magnitudes_whose_r_cubed_leaves_fp32(dtype, cols):
    """Rows of 1e-16, 1e15 and zeros: r^3 is up to 1e51 and down to 1e-45, the
    gradient's terms are all within fp32."""
    x, r, w, dy, ds = make(9, cols, dtype, dtype)
    for rows, size in ((slice(0, 3), 1e-16), (slice(3, 6), 1e15), (slice(6, 7), 0.0)):
        x[rows] *= size
        r[rows] *= size
        ds[rows] /= size or 1.0
    got = api.rms_norm(x, r, w, eps=1e-34)
    assert forward_agrees(got, x, r, w, eps=1e-34)
    for h in (ds, None):
        assert gradient_agrees(api.rms_norm_grad(dy, h, got[1], w, got[2]), dy, h, got[1], w, got[2])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cols,pad,skip", [(64, 8, 0), (64, 8, 8), (64, 3, 1), (13, 5, 2), (2048, 8, 0), (2048, 1, 1)])
def test_row_strides(dtype, cols, pad, skip):
    rows = 37
    big = [torch.randn(rows, cols + pad, device="cuda").to(dtype) for _ in range(6)]
    x, r, y, s, dy, dx = (t[:, skip:skip + cols] for t in big)
    w = torch.randn(cols, device="cuda")
    before = [t.clone() for t in big]
    got = api.rms_norm(x, r, w, out=y, sum_out=s)
    assert got[0].data_ptr() == y.data_ptr() and got[1].data_ptr() == s.data_ptr() and forward_agrees(got, x, r, w)
    grads = api.rms_norm_grad(dy, x, s, w, got[2], out=dx)
    assert gradient_agrees(grads, dy, x, s, w, got[2])
    for i, t in ((2, y), (3, s), (5, dx)):
        before[i][:, skip:skip + cols] = t
    assert all(torch.equal(a, b) for a, b in zip(before, big))     # nothing between the rows was written
    one = torch.randn(1, cols, device="cuda").to(dtype).expand(rows, cols)
    assert forward_agrees(api.rms_norm(x, one, w), x, one, w)
    assert gradient_agrees(api.rms_norm_grad(one, one, s, w, got[2]), one, one, s, w, got[2])
    loose = torch.randn(rows, 1, device="cuda").to(dtype).expand(rows, cols)
    assert gradient_agrees(api.rms_norm_grad(loose, None, s, w, got[2]), loose, None, s, w, got[2])


@pytest.mark.parametrize("cols,pad", [(64, 8), (64, 3), (45, 2), (2048, 16)])
def test_eight_bits_of_and_into_strided_rows(cols, pad):
    big = [torch.randn(21, cols + pad, device="cuda").bfloat16() for _ in range(3)]
    x, r, y = (t[:, :cols] for t in big)
    w, before = torch.randn(cols, device="cuda"), big[2].clone()
    q, scales, s = api.rms_norm_8bit(x, r, w)
    assert eight_agrees(q, scales, forward(x, r, w)[1], cols) and torch.equal(s, forward(x, r, w)[0])
    assert api.decode_8bit(q, scales, out=y).data_ptr() == y.data_ptr()
    before[:, :cols] = api.decode_8bit(q, scales)
    assert torch.equal(before, big[2])
    assert torch.equal(api.decode_8bit(q.view(3, 7, cols), scales.view(3, 7, -1)), y.reshape(3, 7, cols))


@pytest.mark.parametrize("cols", [96, 2048, 40000])
def test_in_place(cols):
    x, r, w, dy, ds = make(5, cols, F32, F32)
    want = api.rms_norm(x, r, w)
    for a, b in (("x", "r"), ("r", "x")):
        t = {"x": x.clone(), "r": r.clone()}
        y, s, rstd = api.rms_norm(t["x"], t["r"], w, out=t[a], sum_out=t[b])
        assert torch.equal(y, want[0]) and torch.equal(s, want[1]) and torch.equal(rstd, want[2])
    grads = api.rms_norm_grad(dy, ds, want[1], w, want[2])
    for name in ("dy", "ds"):
        t = {"dy": dy.clone(), "ds": ds.clone()}
        got = api.rms_norm_grad(t["dy"], t["ds"], want[1], w, want[2], out=t[name])
        assert torch.equal(got[0], grads[0]) and torch.equal(got[1], grads[1])


@pytest.mark.parametrize("cols", [40, 1500])
def test_gradients_by_differences(cols):
    """Central differences of the 64-bit forward along one direction: an error of
    step^2 times the third derivative, which the bound takes from a second step."""
    x, r, w, dy, ds = make(11, cols, F32, F32)
    y, s, rstd = api.rms_norm(x, r, w)
    dx, dw = api.rms_norm_grad(dy, ds, s, w, rstd)
    d, e = torch.randn_like(x).double(), torch.randn_like(w).double()

    def loss(t):
        S = s.double() + t * d
        Y = S * (S.square().mean(1, keepdim=True) + EPS) ** -0.5 * (w.double() + t * e)
        return float((Y * dy.double()).sum() + (S * ds.double()).sum())

    near, far = ((loss(h) - loss(-h)) / (2 * h) for h in (1e-4, 2e-4))
    got = float((dx.double() * d).sum() + (dw.double() * e).sum())
    size = float((dx.double() * d).abs().sum() + (dw.double() * e).abs().sum())
    assert abs(got - near) <= abs(near - far) + (depth(cols) + 30) * U * 4 * size + 1e-9 * abs(loss(0.0)) / 1e-4 * 1e-3


def test_equal_calls_give_equal_bits():
    x, r, w, dy, ds = make(5000, 640, BF, F32)
    y, s, rstd = api.rms_norm(x, r, w)
    first = api.rms_norm_grad(dy, ds, s, w, rstd)
    for _ in range(3):
        again = api.rms_norm_grad(dy, ds, s, w, rstd)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_capture_and_other_streams():
    x, r, w, dy, ds = make(300, 512, BF, F32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, s, rstd = api.rms_norm(x, r, w)
        api.rms_norm_grad(dy, ds, s, w, rstd), api.decode_8bit(*api.rms_norm_8bit(x, r, w)[:2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y, s, rstd = api.rms_norm(x, r, w)
        grads = api.rms_norm_grad(dy, ds, s, w, rstd)
        q, scales, _ = api.rms_norm_8bit(x, r, w)
        back = api.decode_8bit(q, scales)
    for seed in (8, 9):
        for t, n in zip((x, r, w, dy, ds), make(300, 512, BF, F32, seed=seed)):
            t.copy_(n)
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        graph.replay()
        far = api.rms_norm(x, r, w, stream=other.cuda_stream)
        torch.cuda.synchronize()
        assert forward_agrees((y, s, rstd), x, r, w) and gradient_agrees(grads, dy, ds, s, w, rstd)
        assert eight_agrees(q, scales, forward(x, r, w)[1], 512) and torch.equal(far[0], y)
        assert torch.equal(back, api.decode_8bit(q, scales))


def test_offsets_beyond_32_bits():
    rows, cols = (1 << 19) + 5, 4104                       # 2.15e9 elements
    x = torch.zeros(rows, cols, device="cuda", dtype=BF)
    x[-1], x[-2] = 2.0, -3.0
    w = torch.ones(cols, device="cuda", dtype=BF)
    y, s, rstd = api.rms_norm(x, None, w)
    assert s is x and bool((y[-1] == 1).all()) and bool((y[-2] == -1).all()) and float(y[:-2].abs().max()) == 0
    dx, dw = api.rms_norm_grad(y, None, x, w, rstd, out=y)
    assert bool((dw == 2).all())
    assert float(dx[-2:].float().abs().max()) <= 2.0 ** -8 and float(dx[:-2].abs().max()) == 0
    q, scales, _ = api.rms_norm_8bit(x, None, w)
    back = api.decode_8bit(q, scales, out=y)
    assert bool((back[-1] == 1).all()) and bool((back[-2] == -1).all())


def test_zero_sizes_and_refusals():
    w = torch.ones(16, device="cuda")
    e = torch.empty(0, 16, device="cuda")
    assert api.rms_norm(e, None, w)[0].shape == (0, 16)
    dx, dw = api.rms_norm_grad(e, None, e, w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 16) and bool((dw == 0).all())
    assert api.decode_8bit(*api.rms_norm_8bit(e, None, w)[:2]).shape == (0, 16)
    x = torch.ones(4, 16, device="cuda")
    for call in (lambda: api.rms_norm(x.half(), None, w), lambda: api.rms_norm(x.cpu(), None, w), lambda: api.rms_norm(x, x[:2], w),
                 lambda: api.rms_norm(x, None, w[:8]), lambda: api.rms_norm(x, x.bfloat16(), w), lambda: api.rms_norm(x.t(), None, w[:4]),
                 lambda: api.rms_norm_grad(x, None, x, w, w), lambda: api.rms_norm_grad(x[:2], None, x, w, x[:, 0].contiguous()),
                 lambda: api.decode_8bit(x, w), lambda: api.rms_norm(x, None, w.half())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(api.FedOptimaError, match="fp32 or of the tensors' type"):
        api.rms_norm(x, None, w.bfloat16())
    with pytest.raises(api.FedOptimaError, match="eps"):
        api.rms_norm(x, None, w, eps=-1.0)
    with pytest.raises(api.FedOptimaError, match="eps"):
        api.rms_norm(x, None, w, eps=float("nan"))
    with pytest.raises(api.FedOptimaError, match="one tensor"):
        api.rms_norm(x, x, w, out=x, sum_out=x)
    with pytest.raises(api.FedOptimaError, match="stride"):
        api.rms_norm(x, None, w, out=torch.ones(1, 16, device="cuda").expand(4, 16))
