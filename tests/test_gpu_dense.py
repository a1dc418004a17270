"""The operators of include/pconv_dense.h on the GPU against their float64 forms (oracle/dense_oracle.py).

Products are tested twice.  With small whole numbers every sum is exact in 32 bits whatever its order, so the results have to be the
rounded ones bit for bit: nothing is read from a wrong place, left out or counted twice, at any size, stride and alignment.  With real
numbers the curves of the activations and the rounding are tested."""
import numpy as np
import pytest

import paper_2001_07710_amd as pc
from oracle import dense_oracle as D

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16", "bf16"]
CODE = {"f32": pc.F32, "f16": pc.F16, "bf16": pc.BF16}
ACT = {"none": pc.ACT_NONE, "relu": pc.ACT_RELU, "gelu": pc.ACT_GELU, "gelu_tanh": pc.ACT_GELU_TANH, "silu": pc.ACT_SILU}
U32 = 2.0 ** -24
# half a step of the storage type, relative to the value, and the smallest step (of values that underflow)
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}
MARK = -777.0


def say(*a):
    print("[case]", *a, flush=True)


def ttype(dt):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dt]


class Mat:
    """A matrix on the GPU inside a larger buffer: `ahead` elements in front of its first, rows `pad` apart, marked gaps."""

    def __init__(self, a, dt, pad=0, ahead=0):
        import torch
        a = np.asarray(a, np.float64)
        self.rows, self.cols = a.shape
        self.ld, self.dt, self.ahead = self.cols + pad, dt, ahead
        self.buf = torch.full((ahead + self.rows * self.ld + 64,), MARK, dtype=ttype(dt), device="cuda")
        self.view = self.buf[ahead:ahead + self.rows * self.ld].view(self.rows, self.ld)
        self.view[:, :self.cols] = torch.from_numpy(a).cuda().to(ttype(dt))

    def data_ptr(self):
        return self.buf.data_ptr() + self.ahead * self.buf.element_size()

    def get(self):
        """The values; what is around them must be as it was."""
        import torch
        torch.cuda.synchronize()
        rest = self.buf.clone()
        rest[self.ahead:self.ahead + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = MARK
        assert bool((rest == MARK).all()), "a write outside the matrix"
        return self.view[:, :self.cols].double().cpu().numpy()


def empty(rows, cols, dt, pad=0, ahead=0):
    return Mat(np.full((rows, cols), 55.0), dt, pad, ahead)


class Scratch:
    """Workspace of n bytes, filled with NaN, and a mark behind it."""

    def __init__(self, n):
        import torch
        self.n = n
        self.buf = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        self.buf[n:] = 0x5A

    def args(self):
        return {"workspace": self.buf if self.n else None, "workspace_bytes": self.n}

    def check(self):
        assert bool((self.buf[self.n:] == 0x5A).all()), "a write behind the workspace"


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def vec(a):
    import torch
    return None if a is None else torch.from_numpy(np.asarray(a, np.float32)).cuda()


def rounded(a, dt):
    import torch
    return torch.from_numpy(np.asarray(a, np.float64)).to(torch.float32).to(ttype(dt)).double().numpy()


def whole(rng, shape, most):
    return rng.integers(-most, most + 1, shape).astype(np.float64)


# ------------------------------------------------------------------------------------------------------------------ products

# M, N, K: one row and few, sizes around the tiles and stages (64, 128, 256; 32 or 64 of K), lengths of one, many rounds
SIZES = [(1, 1, 1), (1, 17, 64), (3, 40, 500), (16, 130, 1000), (16, 16, 4100), (17, 33, 7), (40, 64, 128), (64, 64, 64), (65, 66, 67),
         (100, 200, 320), (128, 384, 96), (257, 129, 1030), (33, 1000, 2048), (300, 513, 31), (1030, 70, 200)]
LARGE = [(4096, 4096, 72), (4000, 3900, 136)]      # (rounds of the largest tile: whole and ragged)
# elements between rows, elements in front of each matrix: aligned, aligned with gaps, every row at another alignment, an odd start
PLACES = [(0, 0), (8, 16), (3, 0), (0, 1)]


def _linear(x, w, dt, bias, residual, act, first, pad, ahead, keep=True):
    M, K = x.shape
    N = w.shape[0]
    mx, mw, my = Mat(x, dt, pad, ahead), Mat(w, dt, pad, ahead), empty(M, N, dt, pad, ahead)
    mr = None if residual is None else Mat(residual, dt, pad, ahead)
    mz = empty(M, N, dt, pad, ahead) if keep else None
    ws = Scratch(pc.linear_workspace(CODE[dt], M, N, K))
    pc.linear(mx, mw, my, CODE[dt], M, N, K, bias=vec(bias), residual=mr, z=mz, act=ACT[act],
              flags=pc.FLAG_RESIDUAL_FIRST if first else 0, ldx=mx.ld, ldw=mw.ld, ldr=mr.ld if mr else 0, ldy=my.ld, stream=stream(),
              **ws.args())
    y, z = my.get(), mz.get() if keep else None
    ws.check()
    return y, z


@pytest.mark.parametrize("place", PLACES, ids=["tight", "gaps", "odd_rows", "odd_start"])
@pytest.mark.parametrize("dt", TYPES)
def test_linear_is_exact_on_whole_numbers(dt, place):
    rng = np.random.default_rng(10)
    for M, N, K in SIZES + (LARGE if place in ((0, 0), (3, 0)) else []):
        say("linear", dt, place, M, N, K)
        x, w, r = whole(rng, (M, K), 3), whole(rng, (N, K), 2), whole(rng, (M, N), 50)
        b = whole(rng, N, 30)
        # sums stay below 6 * 4,100 + 80 < 2^24, and |z| < 6 * sqrt(K) * 10 far inside fp16's range
        for act, first in (("none", False), ("relu", True), ("relu", False)):
            if act != "none" and M * N > 1 << 20:
                continue
            y, z = _linear(x, w, dt, b, r, act, first, *place)
            yy, zz = D.linear(x, w, b, r, act, first)
            assert np.array_equal(z, rounded(zz, dt)), (dt, place, M, N, K, act, first)
            assert np.array_equal(y, rounded(yy, dt)), (dt, place, M, N, K, act, first)
        if M * N <= 1 << 20:
            y, _ = _linear(x, w, dt, None, None, "none", False, *place, keep=False)
            assert np.array_equal(y, rounded(D.linear(x, w)[0], dt))


def _grad_input(dz, w, dt, z, act, add, pad, ahead):
    M, N = dz.shape
    K = w.shape[1]
    md, mw, mx = Mat(dz, dt, pad, ahead), Mat(w, dt, pad, ahead), empty(M, K, dt, pad, ahead)
    mz, ma = (None if v is None else Mat(v, dt, pad, ahead) for v in (z, add))
    ws = Scratch(pc.linear_grad_input_workspace(CODE[dt], M, N, K))
    pc.linear_grad_input(md, mw, mx, CODE[dt], M, N, K, z=mz, act=ACT[act], add=ma, lddz=md.ld, ldw=mw.ld, ldz=mz.ld if mz else 0,
                         lda=ma.ld if ma else 0, lddx=mx.ld, stream=stream(), **ws.args())
    out = mx.get()
    ws.check()
    return out


def _grad_weight(dz, x, dt, pad, ahead, with_db=True):
    import torch
    M, N = dz.shape
    K = x.shape[1]
    md, mx = Mat(dz, dt, pad, ahead), Mat(x, dt, pad, ahead)
    dw, db = empty(N, K, "f32"), empty(1, N, "f32", 0, ahead)
    ws = Scratch(pc.linear_grad_weight_workspace(CODE[dt], M, N, K))
    pc.linear_grad_weight(md, mx, dw, CODE[dt], M, N, K, db=db if with_db else None, lddz=md.ld, ldx=mx.ld, stream=stream(), **ws.args())
    torch.cuda.synchronize()
    ws.check()
    return dw.get(), db.get()[0]


@pytest.mark.parametrize("place", PLACES, ids=["tight", "gaps", "odd_rows", "odd_start"])
@pytest.mark.parametrize("dt", TYPES)
def test_linear_gradients_are_exact_on_whole_numbers(dt, place):
    rng = np.random.default_rng(11)
    for M, N, K in SIZES + (LARGE if place in ((0, 0), (3, 0)) else []):
        say("gradients", dt, place, M, N, K)
        big = M * K > 1 << 20
        dz, w, x = whole(rng, (M, N), 2), whole(rng, (N, K), 3), whole(rng, (M, K), 3)
        z, add = whole(rng, (M, K), 2), whole(rng, (M, K), 40)
        for act, a in (("none", None), ("relu", add)) if not big else (("relu", None),):
            got = _grad_input(dz, w, dt, z if act != "none" else None, act, a, *place)
            assert np.array_equal(got, rounded(D.linear_grad_input(dz, w, z, act, a), dt)), (dt, place, M, N, K, act)
        dw, db = _grad_weight(dz, x, dt, *place)
        ww, bb = D.linear_grad_weight(dz, x)
        assert np.array_equal(dw, ww) and np.array_equal(db, bb), (dt, place, M, N, K)
    _, db = _grad_weight(dz, x, dt, *place, with_db=False)
    assert (db == 55.0).all()


@pytest.mark.parametrize("place", [(0, 0), (8, 16), (3, 1)], ids=["tight", "gaps", "odd"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_products_of_the_largest_tile_are_exact_on_whole_numbers(dt, place):
    """Results x terms of each product: whole tiles, one for each workgroup; ragged ones, two for some; split along the contraction, the
    last part shorter than the others."""
    rng = np.random.default_rng(12)
    for I, J, C in [(4096, 4096, 512), (4600, 6143, 300), (700, 1300, 16000)]:
        say("largest tile", dt, place, I, J, C)
        # sums stay below 6 * 16,000 + 80 < 2^24, and typical ones, 2 * sqrt(C), are told from their neighbours in either type
        a, b, add = whole(rng, (I, C), 3), whole(rng, (J, C), 2), whole(rng, (I, J), 40)
        bias = whole(rng, J, 30)
        product = a @ b.T
        y, z = _linear(a, b, dt, bias, add, "relu", True, *place)
        zz = product + bias + add
        assert np.array_equal(z, rounded(zz, dt)) and np.array_equal(y, rounded(np.maximum(zz, 0), dt)), (dt, place, I, J, C)
        got = _grad_input(a, np.ascontiguousarray(b.T), dt, add, "relu", add, *place)
        assert np.array_equal(got, rounded(np.where(add > 0, product, 0) + add, dt)), (dt, place, I, J, C)
        dw, db = _grad_weight(np.ascontiguousarray(a.T), np.ascontiguousarray(b.T), dt, *place)
        assert np.array_equal(dw, product) and np.array_equal(db, a.sum(1)), (dt, place, I, J, C)


def _close(got, want, dt, slack):
    """|got - want| within the rounding of the stored result and `slack` for what 32-bit arithmetic before it may be off."""
    bound = HALF[dt] * np.abs(want) + TINY[dt] + slack * (1 + HALF[dt])
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (dt, int(bad.sum()), float(np.max((np.abs(got - want) / bound)[bad])))


@pytest.mark.parametrize("dt", TYPES)
def test_the_tail_of_gelu(dt):
    """Relative to the tail itself: its curve to 20 units of 2^-24 with about as many for the evaluation (fp32: erfc to 16), the argument of
    the exponential to t^2 / 2 * 2 units (t is rounded into it twice), one for each other product: (t^2 + 64) units."""
    from math import erfc, sqrt
    v = rounded(-np.linspace(0, 8, 3001), dt)[:, None]
    y, z = _linear(v, np.ones((1, 1)), dt, None, None, "gelu", False, 0, 0)
    assert np.array_equal(z, v)
    want = v * np.vectorize(lambda t: erfc(-t / sqrt(2)) / 2)(v)
    _close(y, want, dt, (v * v + 64) * U32 * np.abs(want))


def _tail(act, v):
    """(curve, slope, what the slope's rounding errors are relative to) at v <= 0, without cancellation; v as far as fp32 has the curve."""
    from math import erfc, sqrt
    if act == "gelu":
        s = np.vectorize(lambda t: erfc(-t / sqrt(2)) / 2)(v)
        rise = v * np.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    else:
        c = 2 * np.sqrt(2 / np.pi)
        u, du = (v, 1.0) if act == "silu" else (c * (v + 0.044715 * v ** 3), c * (1 + 3 * 0.044715 * v * v))
        s = 1 / (1 + np.exp(-u))
        rise = v * s / (1 + np.exp(u)) * du
    return v * s, s + rise, s + np.abs(rise)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dt", TYPES)
def test_the_tails_of_activations_and_of_their_slopes(dt, act):
    """Relative to the tail itself, in units of 2^-24.  fp32: the exponential 2, its argument's remainder 1, 1 + e 1, the reciprocal 2, z times
    it 1 (GELU: erfc 16, half of the slope's product 2): 8 and 20; the slope's factors and sum 8 more.  16 bits: the exponent x rounded up to
    three times costs 3 |x| units, the polynomial of GELU's tail 20, the other roundings 16."""
    far = {"gelu": 12.5, "gelu_tanh": 9.5, "silu": 80.0}[act]
    v = rounded(-np.linspace(0, far, 4001), dt)[:, None]
    y, z = _linear(v, np.ones((1, 1)), dt, None, None, act, False, 0, 0)
    assert np.array_equal(z, v)
    curve, slope, size = _tail(act, v)
    x = np.abs({"gelu": v * v / 2, "gelu_tanh": 1.6 * (v + 0.044715 * v ** 3), "silu": v}[act])
    units = (20 if act == "gelu" else 8) if dt == "f32" else 3 * x + 36
    _close(y, curve, dt, units * U32 * np.abs(curve))
    one, mv, mo = Mat(np.ones(v.shape), dt), Mat(v, dt), empty(*v.shape, dt)
    pc.activation_grad(one, mv, mo, CODE[dt], *v.shape, ACT[act], stream=stream())
    _close(mo.get(), slope, dt, (units + 8) * U32 * size)


@pytest.mark.parametrize("act", D.ACTS)
@pytest.mark.parametrize("dt", TYPES)
def test_activations_and_their_slopes(dt, act):
    """z comes out exactly (whole numbers over 16), so y is the curve of a known argument.  The curves and slopes are evaluated in 32 bits: an
    error of a few units there (exp and erf to 2 ulp, the argument of exp to |argument| <= 25 where its result counts, sums of terms of
    at most 1.2 |z| + 1): 64 * 2^-24 relative to |z| + 1 covers 25 + 2 units of exp's argument and the sums' terms twice over."""
    rng = np.random.default_rng(12)
    M, N, K = 40, 72, 16
    x, w = whole(rng, (M, K), 3) / 4, whole(rng, (N, K), 3) / 4
    r = whole(rng, (M, N), 64) / 16
    for first in (False, True):
        y, z = _linear(x, w, dt, None, r, act, first, 0, 0)
        yy, zz = D.linear(x, w, None, r, act, first)
        assert np.array_equal(z, zz) or dt == "bf16"
        _close(y, yy, dt, 64 * U32 * (np.abs(zz) + np.abs(r) + 1))
    v = np.concatenate([np.linspace(-12, 12, 997), [0.0, -0.0, 1e-6, -1e-6, 60000.0, -60000.0]])
    v = rounded(v, dt)[None, :].repeat(3, 0)
    g = rounded(rng.standard_normal(v.shape), dt)
    for pad, ahead in PLACES:
        mg, mv, mo = Mat(g, dt, pad, ahead), Mat(v, dt, pad, ahead), empty(*v.shape, dt, pad, ahead)
        pc.activation_grad(mg, mv, mo, CODE[dt], *v.shape, ACT[act], lddy=mg.ld, ldz=mv.ld, lddz=mo.ld, stream=stream())
        with np.errstate(over="ignore"):
            want = g * D.act_slope(v, act)
        _close(mo.get(), want, dt, 64 * U32 * np.abs(g) * (np.minimum(np.abs(v), 13) + 1))
    # the same slopes behind a product that hands its operand through
    z = rounded(rng.standard_normal((M, N)) * 3, dt)
    dz = rounded(rng.standard_normal((M, N)), dt)
    add = rounded(rng.standard_normal((M, N)), dt)
    got = _grad_input(dz, np.eye(N), dt, z if act != "none" else None, act, add, 0, 0)
    want = D.linear_grad_input(dz, np.eye(N), z, act, add)
    _close(got, want, dt, 64 * U32 * ((np.abs(z) + 1) * np.abs(dz) + np.abs(add)))


@pytest.mark.parametrize("act", D.ACTS)
def test_activations_of_extreme_arguments(act):
    z = np.array([[np.inf, -np.inf, np.nan, 3e38, -3e38, 65504.0, -65504.0, 0.0]])
    mz, mo, one = Mat(z, "f32"), empty(1, 8, "f32"), Mat(np.ones((1, 8)), "f32")
    pc.activation_grad(one, mz, mo, pc.F32, 1, 8, ACT[act], stream=stream())
    got = mo.get()[0]
    want = {"none": [1, 1, 1, 1, 1, 1, 1, 1], "relu": [1, 0, np.nan, 1, 0, 1, 0, 0]}.get(act, [1, 0, np.nan, 1, 0, 1, 0, 0.5])
    assert np.allclose(got, want, rtol=0, atol=1e-30, equal_nan=True), got
    y, _ = _linear(np.array([[1.0]]), np.array([[1.0]]), "f32", None, None, act, False, 0, 0)
    big, _ = _linear(np.array([[3e38], [-3e38], [np.nan], [np.inf]]), np.array([[1.0]]), "f32", None, None, act, False, 0, 0)
    assert big[0, 0] == np.float32(3e38) and np.isnan(big[2, 0]) and big[3, 0] == np.inf
    assert big[1, 0] == (np.float32(-3e38) if act == "none" else 0) or abs(big[1, 0]) <= 1e-4


@pytest.mark.parametrize("dt", TYPES)
def test_products_of_real_numbers(dt):
    """Random signs: the error of a sum of K products in 32 bits is a random walk of K steps of at most half a unit of the running sum,
    whose size is below sqrt(K) |x| |w|; six times sqrt(K) / 2 steps of it, and K |x||w| units at the very most, are allowed."""
    rng = np.random.default_rng(13)
    for M, N, K in [(1, 1000, 512), (5, 300, 3000), (200, 300, 1000), (1000, 260, 4096)]:
        say("real", dt, M, N, K)
        x, w = rounded(rng.standard_normal((M, K)), dt), rounded(rng.standard_normal((N, K)) / np.sqrt(K), dt)
        y, _ = _linear(x, w, dt, None, None, "none", False, 0, 0, keep=False)
        size = np.sqrt((x * x) @ (w * w).T)                       # the running sum's size at its end
        _close(y, x @ w.T, dt, 6 * U32 * np.sqrt(K) * size)
        dw, db = _grad_weight(x, x[:, :min(K, 500)], dt, 0, 0)
        ww, bb = D.linear_grad_weight(x, x[:, :min(K, 500)])
        size = np.sqrt((x * x).T @ (x * x)[:, :min(K, 500)])
        assert (np.abs(dw - ww) <= 6 * U32 * np.sqrt(M) * size + M * U32 * np.abs(ww)).all()
        assert (np.abs(db - bb) <= 6 * U32 * np.sqrt(M) * np.sqrt((x * x).sum(0))).all()


@pytest.mark.parametrize("dt", TYPES)
def test_a_row_does_not_depend_on_its_place_nor_on_its_neighbours(dt):
    """Equal rows give equal results, and non-finite values stay in their row (and, of w, in their column)."""
    rng = np.random.default_rng(14)
    for M, N, K in [(9, 50, 300), (150, 140, 203), (400, 700, 264)]:
        x, w = rounded(rng.standard_normal((1, K)), dt).repeat(M, 0), rounded(rng.standard_normal((N, K)), dt)
        y, _ = _linear(x, w, dt, None, None, "none", False, 0, 0)
        assert (y == y[0]).all()
        x[3, 5], x[M - 1, K - 1] = np.inf, np.nan
        w[N - 2, 0] = np.nan
        z, _ = _linear(x, w, dt, None, None, "none", False, 0, 0)
        clean = np.ones((M, N), bool)
        clean[[3, M - 1]] = False
        clean[:, N - 2] = False
        assert np.array_equal(z[clean], y[clean]) and not np.isfinite(z[:, N - 2]).any() and not np.isfinite(z[3]).any()


# M, N, K: the smallest tile, whole and ragged; the same split; few rows, split; the middle tile; the largest, two for some workgroups
ALIKE = [(150, 140, 203), (192, 128, 256), (100, 130, 5000), (9, 70, 3000), (2100, 2200, 136), (4600, 6143, 200)]


@pytest.mark.parametrize("act", D.ACTS)
@pytest.mark.parametrize("dt", TYPES)
def test_equal_rows_give_equal_results_in_every_epilogue(dt, act):
    """Rows of whole and of ragged tiles leave by different ways, and rows of a window by different lanes: all the same, to the bit."""
    import torch
    rng = np.random.default_rng(16)
    for M, N, K in ALIKE if act in ("none", "gelu") else ALIKE[:-1]:
        alike = lambda n: torch.from_numpy(rounded(rng.standard_normal((1, n)), dt)).cuda().to(ttype(dt)).repeat(M, 1)  # noqa: E731
        x, r, add, w = alike(K), alike(N), alike(K), vec(rng.standard_normal((N, K)) / np.sqrt(K)).to(ttype(dt))
        bias = vec(rng.standard_normal(N))
        say("alike", dt, act, M, N, K)
        ws = Scratch(max(pc.linear_workspace(CODE[dt], M, N, K), pc.linear_grad_input_workspace(CODE[dt], M, N, K)))
        for residual, flags, keep in ((None, 0, False), (r, 0, True), (r, pc.FLAG_RESIDUAL_FIRST, True), (r, pc.FLAG_RESIDUAL_FIRST, False)):
            y, z = torch.full((M, N), 55.0, dtype=ttype(dt), device="cuda"), torch.full((M, N), 55.0, dtype=ttype(dt), device="cuda")
            pc.linear(x, w, y, CODE[dt], M, N, K, bias=bias, residual=residual, z=z if keep else None, act=ACT[act], flags=flags,
                      stream=stream(), **ws.args())
            assert bool((y == y[0]).all()) and bool((z == z[0]).all()), (dt, act, M, N, K, flags, keep)
        for more in (None, add):
            dx = torch.full((M, K), 55.0, dtype=ttype(dt), device="cuda")
            pc.linear_grad_input(r, w, dx, CODE[dt], M, N, K, z=x if act != "none" else None, act=ACT[act], add=more, stream=stream(),
                                 **ws.args())
            assert bool((dx == dx[0]).all()), (dt, act, M, N, K)
        ws.check()


@pytest.mark.parametrize("dt", TYPES)
def test_arguments_of_activations_are_kept_exactly(dt):
    """z of whole sixteenths, 9 + 4 at most: 208 of them, which eight bits hold."""
    rng = np.random.default_rng(17)
    x, w, r = whole(rng, (40, 16), 3) / 4, whole(rng, (72, 16), 3) / 4, whole(rng, (40, 72), 64) / 16
    for act in D.ACTS:
        for first in (False, True):
            _, z = _linear(x, w, dt, None, r, act, first, 0, 0)
            assert np.array_equal(z, D.linear(x, w, None, r, act, first)[1]), (dt, act, first)


# (elements between rows, elements in front) of every matrix, each its own: all rows aligned; the first, the second operand alone not; neither
APART = [[(8, 0), (16, 8), (24, 16), (32, 0), (40, 8)], [(3, 1), (16, 8), (5, 0), (0, 0), (9, 2)], [(8, 16), (7, 0), (2, 5), (11, 3), (0, 8)],
         [(1, 3), (5, 1), (0, 2), (13, 0), (6, 7)]]


@pytest.mark.parametrize("places", APART, ids=["aligned", "first", "second", "neither"])
@pytest.mark.parametrize("dt", TYPES)
def test_every_matrix_has_a_stride_of_its_own(dt, places):
    """Square products, so that a stride taken for another's stays inside the matrices' buffers or reads marks; whole numbers, to the bit."""
    import torch
    rng = np.random.default_rng(18)
    for n in (24, 200, 264):
        say("apart", dt, n)
        a, b, c, d = (whole(rng, (n, n), 3) for _ in range(4))
        bias = whole(rng, n, 20)
        ma, mb, mc, md, mo = ([Mat(v, dt, *at) for v, at in zip((a, b, c, d), places)] + [empty(n, n, dt, *places[4])])
        mz = empty(n, n, dt, places[4][0], 3)
        ws = Scratch(max(f(CODE[dt], n, n, n) for f in (pc.linear_workspace, pc.linear_grad_input_workspace, pc.linear_grad_weight_workspace)))
        pc.linear(ma, mb, mo, CODE[dt], n, n, n, bias=vec(bias), residual=mc, z=mz, act=pc.ACT_RELU, ldx=ma.ld, ldw=mb.ld, ldr=mc.ld,
                  ldy=mo.ld, stream=stream(), **ws.args())
        y, z = D.linear(a, b, bias, c, "relu", False)
        assert np.array_equal(mo.get(), rounded(y, dt)) and np.array_equal(mz.get(), rounded(z, dt))
        pc.linear_grad_input(ma, mb, mo, CODE[dt], n, n, n, z=mc, act=pc.ACT_RELU, add=md, lddz=ma.ld, ldw=mb.ld, ldz=mc.ld, lda=md.ld,
                             lddx=mo.ld, stream=stream(), **ws.args())
        assert np.array_equal(mo.get(), rounded(D.linear_grad_input(a, b, c, "relu", d), dt))
        dw, db = empty(n, n, "f32"), empty(1, n, "f32")
        pc.linear_grad_weight(ma, mb, dw, CODE[dt], n, n, n, db=db, lddz=ma.ld, ldx=mb.ld, stream=stream(), **ws.args())
        want = D.linear_grad_weight(a, b)
        assert np.array_equal(dw.get(), want[0]) and np.array_equal(db.get()[0], want[1])
        pc.activation_grad(ma, mb, mo, CODE[dt], n, n, pc.ACT_RELU, lddy=ma.ld, ldz=mb.ld, lddz=mo.ld, stream=stream())
        assert np.array_equal(mo.get(), a * (b > 0))
        ws.check()
        # layer norm at strides of their own is layer norm at one: the same rows tightly packed, to the bit
        ta, tb, to = Mat(a, dt), Mat(b, dt), empty(n, n, dt)
        stats = [[torch.empty(n, device="cuda") for _ in range(2)] for _ in range(2)]
        out = [[empty(1, n, "f32") for _ in range(2)] for _ in range(2)]
        need = pc.layer_norm_grad_workspace(CODE[dt], n, n)
        for (mx, mdy, my), (mean, rstd), (dg, dbeta) in zip(((ma, mb, mo), (ta, tb, to)), stats, out):
            pc.layer_norm(mx, my, CODE[dt], n, n, gamma=vec(bias), beta=vec(bias), mean=mean, rstd=rstd, ldx=mx.ld, ldy=my.ld, stream=stream())
            first = my.get()
            ws = Scratch(need)
            pc.layer_norm_grad(mdy, mx, my, mean, rstd, CODE[dt], n, n, gamma=vec(bias), dgamma=dg, dbeta=dbeta, lddy=mdy.ld, ldx=mx.ld,
                               lddx=my.ld, stream=stream(), **ws.args())
            second = my.get()
            if mx is ma:
                y, dx = first, second
        assert y.tobytes() == first.tobytes() and dx.tobytes() == second.tobytes()
        for one, other in zip(out[0] + [empty(1, 1, "f32")], out[1] + [empty(1, 1, "f32")]):
            assert one.get().tobytes() == other.get().tobytes()
        assert all(torch.equal(p, q) for p, q in zip(*stats))


@pytest.mark.parametrize("dt", TYPES)
def test_products_of_rows_that_lie_2_to_the_20_elements_apart(dt):
    """The longest stride there is, in every matrix, at the smallest and (16 bits) the largest tile: offsets inside a tile pass 2^28 bytes."""
    import torch
    rng = np.random.default_rng(19)
    ld = 1 << 20
    for M, N, K in [(70, 90, 200), (5, 40, 333)] + ([(4096, 4096, 72)] if dt == "f16" else []):
        say("far rows", dt, M, N, K)
        x, w, r = whole(rng, (M, K), 3), whole(rng, (N, K), 2), whole(rng, (M, N), 30)

        def far(a):
            t = torch.empty((a.shape[0], ld), dtype=ttype(dt), device="cuda")[:, :a.shape[1]]
            t.copy_(torch.from_numpy(a).cuda())
            return t
        fx, fw, fr, fy = far(x), far(w), far(r), far(np.full((M, N), 55.0))
        ws = Scratch(max(f(CODE[dt], M, N, K) for f in (pc.linear_workspace, pc.linear_grad_input_workspace, pc.linear_grad_weight_workspace)))
        pc.linear(fx, fw, fy, CODE[dt], M, N, K, residual=fr, ldx=ld, ldw=ld, ldr=ld, ldy=ld, stream=stream(), **ws.args())
        assert np.array_equal(fy.double().cpu().numpy(), rounded(x @ w.T + r, dt))
        pc.linear_grad_input(fr, fw, fx, CODE[dt], M, N, K, lddz=ld, ldw=ld, lddx=ld, stream=stream(), **ws.args())
        assert np.array_equal(fx.double().cpu().numpy(), rounded(r @ w, dt))
        fx.copy_(torch.from_numpy(x).cuda())
        dw, db = empty(N, K, "f32"), empty(1, N, "f32")
        pc.linear_grad_weight(fr, fx, dw, CODE[dt], M, N, K, db=db, lddz=ld, ldx=ld, stream=stream(), **ws.args())
        assert np.array_equal(dw.get(), r.T @ x) and np.array_equal(db.get()[0], r.sum(0))
        ws.check()


@pytest.mark.parametrize("dt", TYPES)
def test_few_rows_whose_long_sums_are_shared_are_exact_on_whole_numbers(dt):
    rng = np.random.default_rng(23)
    for M, N, K in [(1, 16, 20000), (5, 200, 9001), (16, 1000, 12000), (2, 2001, 8192), (7, 70, 4097)]:
        say("few rows", dt, M, N, K)
        assert pc.linear_workspace(CODE[dt], M, N, K) > 0
        # sums stay below 6 * 20,000 + 80 < 2^24 and, 2 * sqrt(K) each, far inside fp16's range
        x, w, r, b = whole(rng, (M, K), 3), whole(rng, (N, K), 2), whole(rng, (M, N), 50), whole(rng, N, 30)
        for place in ((0, 0), (8, 16), (3, 1)):
            y, z = _linear(x, w, dt, b, r, "relu", True, *place)
            yy, zz = D.linear(x, w, b, r, "relu", True)
            assert np.array_equal(z, rounded(zz, dt)) and np.array_equal(y, rounded(yy, dt)), (dt, place, M, N, K)


def test_products_run_twice_alike_and_in_place():
    import torch
    rng = np.random.default_rng(15)
    M, N, K = 64, 300, 5000                         # (split: parts meet in the workspace)
    x, w, r = (rounded(rng.standard_normal(s), "bf16") for s in ((M, K), (N, K), (M, N)))
    assert pc.linear_workspace(pc.BF16, M, N, K) > 0
    a, _ = _linear(x, w, "bf16", None, r, "silu", False, 0, 0)
    b, _ = _linear(x, w, "bf16", None, r, "silu", False, 0, 0)
    assert a.tobytes() == b.tobytes()
    mx, mw, mr = Mat(x, "bf16"), Mat(w, "bf16"), Mat(r, "bf16")
    ws = Scratch(pc.linear_workspace(pc.BF16, M, N, K))
    pc.linear(mx, mw, mr, pc.BF16, M, N, K, residual=mr, act=pc.ACT_SILU, stream=stream(), **ws.args())     # the residual is y
    assert mr.get().tobytes() == a.tobytes()
    dz = rounded(rng.standard_normal((M, N)), "bf16")
    want = _grad_input(dz, w, "bf16", None, "none", x, 0, 0)
    md, ma = Mat(dz, "bf16"), Mat(x, "bf16")
    ws = Scratch(pc.linear_grad_input_workspace(pc.BF16, M, N, K))
    pc.linear_grad_input(md, mw, ma, pc.BF16, M, N, K, add=ma, stream=stream(), **ws.args())                # add is dx
    assert ma.get().tobytes() == want.tobytes()
    v, g = Mat(x, "bf16"), Mat(w[:M] if N >= M else x, "bf16")
    pc.activation_grad(g, v, g, pc.BF16, M, K, pc.ACT_GELU, stream=stream())                                # dz is dy
    o = empty(M, K, "bf16")
    pc.activation_grad(Mat(w[:M], "bf16"), v, o, pc.BF16, M, K, pc.ACT_GELU, stream=stream())
    assert g.get().tobytes() == o.get().tobytes()
    torch.cuda.synchronize()


def test_no_rows():
    dw, db, ws = empty(5, 6, "f32"), empty(1, 5, "f32"), Scratch(0)
    pc.linear_grad_weight(None, None, dw, pc.F16, 0, 5, 6, db=db, stream=stream(), **ws.args())
    assert not dw.get().any() and not db.get().any()
    dg, db = empty(1, 40, "f32"), empty(1, 40, "f32")
    pc.layer_norm_grad(None, None, None, None, None, pc.F16, 0, 40, dgamma=dg, dbeta=db, stream=stream())
    assert not dg.get().any() and not db.get().any()


# ---------------------------------------------------------------------------------------------------------------- layer norm

# every spread of a row over threads, in either element size, one element more and less; rows longer than a workgroup holds
WIDTHS = [1, 2, 7, 8, 16, 31, 33, 64, 100, 129, 200, 256, 257, 500, 512, 1000, 1024, 1025, 2047, 2049, 4096, 4100, 8192, 8195, 16384, 20000,
          32768, 32769, 40001]


@pytest.mark.parametrize("place", PLACES, ids=["tight", "gaps", "odd_rows", "odd_start"])
@pytest.mark.parametrize("dt", TYPES)
def test_layer_norm_forward_and_backward(dt, place):
    """Mean and variance are sums of D values in 32 bits over a tree: an error of log2(D) + the 32 values that a thread adds in a row,
    below 64 units, relative to the root mean square; the mean's comes back in x - mean, once, and rstd's as a factor.  Backward the two
    means carry the same, times |g| and |g h|."""
    import torch
    rng = np.random.default_rng(20)
    pad, ahead = place
    for Dn in WIDTHS if place in ((0, 0), (0, 1)) else WIDTHS[::3]:
        rows = int(rng.integers(1, 40)) if Dn > 600 else int(rng.integers(1, 700))
        say("norm", dt, place, rows, Dn)
        x = rounded(rng.standard_normal((rows, Dn)) * 1.5 + 0.5, dt)
        dy = rounded(rng.standard_normal((rows, Dn)), dt)
        gamma, beta = (rng.standard_normal(Dn).astype(np.float32) for _ in range(2))
        eps = 1e-2 if Dn < 8 else 1e-5
        mx, my = Mat(x, dt, pad, ahead), empty(rows, Dn, dt, pad, ahead)
        mean, rstd = empty(1, rows, "f32"), empty(1, rows, "f32")
        pc.layer_norm(mx, my, CODE[dt], rows, Dn, gamma=vec(gamma), beta=vec(beta), eps=eps, mean=mean, rstd=rstd, ldx=mx.ld, ldy=my.ld,
                      stream=stream())
        y, m, s = D.layer_norm(x, gamma, beta, eps)
        rms = np.sqrt((x * x).mean(1)) + 1e-30
        assert (np.abs(mean.get()[0] - m) <= 64 * U32 * rms).all()
        assert (np.abs(rstd.get()[0] - s) <= 64 * U32 * s * (1 + (rms * s) ** 2)).all()
        off = 64 * U32 * (rms * s)[:, None]                                   # of h
        h = (x - m[:, None]) * s[:, None]
        _close(my.get(), y, dt, (off + 192 * U32 * np.abs(h)) * np.abs(gamma) + 4 * U32 * (np.abs(beta) + np.abs(y)))
        md, mo = Mat(dy, dt, pad, ahead), empty(rows, Dn, dt, pad, ahead)
        dg, db = empty(1, Dn, "f32"), empty(1, Dn, "f32")
        ws = Scratch(pc.layer_norm_grad_workspace(CODE[dt], rows, Dn))
        pc.layer_norm_grad(md, mx, mo, mean, rstd, CODE[dt], rows, Dn, gamma=vec(gamma), dgamma=dg, dbeta=db, lddy=md.ld, ldx=mx.ld,
                           lddx=mo.ld, stream=stream(), **ws.args())
        dx, dgamma, dbeta = D.layer_norm_grad(dy, x, gamma, eps)
        ws.check()
        g = np.abs(dy * gamma)
        rg, rh = np.sqrt((g * g).mean(1))[:, None], np.sqrt(((g * h) ** 2).mean(1))[:, None]
        slack = s[:, None] * (64 * U32 * (rg + np.abs(h) * rh + g) + (off + 192 * U32 * np.abs(h)) * (rh + rg + 1) + off * np.abs(h) * rg)
        _close(mo.get(), dx, dt, slack + 192 * U32 * np.abs(dx))
        size = np.sqrt((dy * dy * (h * h + 1)).sum(0))
        assert (np.abs(dg.get()[0] - dgamma) <= 6 * U32 * np.sqrt(rows + 64) * size + (np.abs(dy) * (off + 192 * U32 * np.abs(h))).sum(0)).all()
        assert (np.abs(db.get()[0] - dbeta) <= 6 * U32 * np.sqrt(rows + 64) * size).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,Dn", [(5000, 64), (9000, 16), (4000, 200), (3000, 1024), (2500, 4096), (1200, 40000)])
def test_column_sums_of_many_rows_are_exact_on_whole_numbers(rows, Dn):
    """x - mean = +-1 and rstd = 1 by construction (half of a row 0, half 2, statistics given): every term is whole."""
    rng = np.random.default_rng(21)
    x = np.where(np.arange(Dn) % 2 == 0, 0.0, 2.0)[None, :].repeat(rows, 0)
    dy = whole(rng, (rows, Dn), 3)
    mx, md, mo = Mat(x, "bf16"), Mat(dy, "bf16"), empty(rows, Dn, "bf16")
    one, dg, db = vec(np.ones(rows)), empty(1, Dn, "f32"), empty(1, Dn, "f32")
    n = pc.layer_norm_grad_workspace(pc.BF16, rows, Dn)
    for asked in ({"dgamma": dg, "dbeta": db}, {"dgamma": dg}, {"dbeta": db}):
        dg.view.fill_(5.0), db.view.fill_(5.0)
        ws = Scratch(n)
        pc.layer_norm_grad(md, mx, mo if len(asked) == 2 else None, one, one, pc.BF16, rows, Dn, stream=stream(), **asked, **ws.args())
        h = x - 1.0
        assert np.array_equal(dg.get()[0], (dy * h).sum(0) if "dgamma" in asked else np.full(Dn, 5.0))
        assert np.array_equal(db.get()[0], dy.sum(0) if "dbeta" in asked else np.full(Dn, 5.0))
        ws.check()
    got = mo.get()
    pc.layer_norm_grad(md, mx, mo, one, one, pc.BF16, rows, Dn, stream=stream())                    # dx alone, no workspace
    assert mo.get().tobytes() == got.tobytes()
    pc.layer_norm_grad(md, mx, md, one, one, pc.BF16, rows, Dn, stream=stream())                    # dx is dy
    assert md.get().tobytes() == got.tobytes()


@pytest.mark.parametrize("dt", TYPES)
def test_layer_norm_without_weights_in_place_and_of_equal_values(dt):
    rng = np.random.default_rng(22)
    x = rounded(rng.standard_normal((50, 300)), dt)
    x[7] = 0.5                                                        # no variance: zeros
    mx, my = Mat(x, dt), empty(50, 300, dt)
    pc.layer_norm(mx, my, CODE[dt], 50, 300, stream=stream())
    y = my.get()
    assert not y[7].any()
    _close(y, D.layer_norm(x)[0], dt, 256 * U32 * (np.abs(D.layer_norm(x)[0]) + 1))
    pc.layer_norm(mx, mx, CODE[dt], 50, 300, stream=stream())
    assert mx.get().tobytes() == y.tobytes()
    x[3, 5], x[4, 299] = np.inf, np.nan                               # stay in their rows
    mx = Mat(x, dt)
    pc.layer_norm(mx, my, CODE[dt], 50, 300, stream=stream())
    z, rest = my.get(), np.delete(np.arange(50), [3, 4])
    assert z[rest].tobytes() == y[rest].tobytes() and np.isnan(z[4]).all() and np.isnan(z[3, 5])


@pytest.mark.parametrize("dt", TYPES)
def test_layer_norm_of_rows_of_equal_values_is_exact(dt):
    """Rows of one value, at every spread of a row over threads.  The first mean is off by k units of the value's last place: a sum of 16-bit
    values is exact but for its last additions (k <= 10), one of fp32 values passes 36 additions, then comes a product with 1 / D (k <= 38).  All deviations are
    then that k, exactly, and their sum and their squares' are whole multiples below 2^24 units (38^2 * 8,200 = 1.2e7): the mean is the value,
    the variance 0 and y beta.  rstd: a root, a quotient and eps, two units each."""
    rng = np.random.default_rng(24)
    levels = rounded(np.array([0.1, 100, 1000, 4000, 30000, -777, 1 / 3, -61000.0]), dt)
    for Dn in (26, 41, 100, 200, 500, 1000, 1025, 2000, 4001, 8191, 8200, 16383, 16400):
        if dt == "f32" and Dn > 8200:
            continue
        rows = 5 * len(levels) if Dn < 600 else len(levels)
        x = levels[np.arange(rows) % len(levels)][:, None].repeat(Dn, 1)
        gamma, beta = (rng.standard_normal(Dn).astype(np.float32) for _ in range(2))
        say("equal values", dt, rows, Dn)
        for eps in (1e-5, 0.0) if Dn <= 1025 else (1e-5,):
            mx, my, mean, rstd = Mat(x, dt), empty(rows, Dn, dt), empty(1, rows, "f32"), empty(1, rows, "f32")
            pc.layer_norm(mx, my, CODE[dt], rows, Dn, gamma=vec(gamma), beta=vec(beta), eps=eps, mean=mean, rstd=rstd, stream=stream())
            assert np.array_equal(mean.get()[0], x[:, 0]), (dt, Dn, eps)
            if eps:
                assert np.array_equal(my.get(), rounded(beta, dt)[None, :].repeat(rows, 0)), (dt, Dn)
                want = 1 / np.sqrt(float(np.float32(eps)))
                assert (np.abs(rstd.get()[0] - want) <= 6 * U32 * want).all(), (dt, Dn)
            else:                                                      # 0 / 0, like the formula
                assert np.isnan(my.get()).all() and np.isinf(rstd.get()[0]).all(), (dt, Dn)


@pytest.mark.parametrize("dt", TYPES)
def test_layer_norm_of_rows_far_from_zero(dt):
    """Rows whose spread is small against their level: x - mean is exact around the first mean, so that everything behind it is relative to
    the spread, sums of 64 units as in the test above of rows near zero; the first mean, 40 units of the level off at most, is less than half
    of the spread away, whose square is a quarter of the variance that is taken off again: 128 units for the mean, 192 |h| for rstd."""
    rng = np.random.default_rng(25)
    step = {"f32": 2.0 ** -6, "f16": 0.5, "bf16": 4.0}[dt]
    for Dn in (41, 100, 300, 1000, 2000, 4001, 8191, 16383, 40000):
        rows = 30 if Dn < 600 else 6
        x = 1000.0 + step * (rng.integers(-2, 3, (rows, Dn)) if dt == "f32" else rng.random((rows, Dn)) < 0.1)
        gamma = rng.standard_normal(Dn).astype(np.float32)
        say("far from zero", dt, rows, Dn)
        assert np.array_equal(rounded(x, dt), x)
        mx, my, mean, rstd = Mat(x, dt), empty(rows, Dn, dt), empty(1, rows, "f32"), empty(1, rows, "f32")
        pc.layer_norm(mx, my, CODE[dt], rows, Dn, gamma=vec(gamma), mean=mean, rstd=rstd, stream=stream())
        y, m, s = D.layer_norm(x, gamma, None, float(np.float32(1e-5)))
        h = (x - m[:, None]) * s[:, None]
        assert (np.abs(mean.get()[0] - m) <= U32 * np.abs(m) + 64 * U32 / s).all(), (dt, Dn)
        assert (np.abs(rstd.get()[0] - s) <= 96 * U32 * s).all(), (dt, Dn)
        _close(my.get(), y, dt, (128 + 192 * np.abs(h)) * U32 * np.abs(gamma) + 4 * U32 * np.abs(y))


# -------------------------------------------------------------------------------------------------------------- distillation

def _distill(s, idx, val, dt, T, weight=None, pad=0, ahead=0, gpad=None, gahead=None, what=("loss", "grad", "stats")):
    import torch
    R, V = s.shape
    ms = Mat(s, dt, pad, ahead)
    mg = empty(R, V, dt, pad if gpad is None else gpad, ahead if gahead is None else gahead)
    loss, stats = empty(1, R, "f32"), empty(R, 2, "f32")
    i, v = torch.from_numpy(np.asarray(idx, np.int32)).cuda(), vec(val)
    pc.distill(ms, i, v, CODE[dt], R, V, i.shape[1], T, weight=vec(weight), loss=loss if "loss" in what else None,
               grad=mg if "grad" in what else None, stats=stats if "stats" in what else None, ldl=ms.ld, ldg=mg.ld, stream=stream())
    return loss.get()[0], mg.get(), stats, ms, i, v


def _distill_bounds(s, idx, val, T, w):
    """Errors of 32-bit arithmetic: an exponential's argument d / T, |d| / T <= 100 where its result counts, is off by two units of it,
    exp and log by two units, the sums over V by log2(V) + 32 < 64 units: relative to q, 64 + 2 * |d| / T + 8 units; the loss adds terms
    p * (log p - log q), each to 8 units of |log p| + |log q| + the sums' 64."""
    z = s / T
    d = np.abs(z - z.max(1, keepdims=True))
    q = np.exp(z - z.max(1, keepdims=True))
    q = q / q.sum(1, keepdims=True)
    t = np.where(idx >= 0, val / T, -np.inf)
    with np.errstate(invalid="ignore"):
        td = np.where(idx >= 0, np.abs(t - t.max(1, keepdims=True)), 0)
        p = np.exp(t - t.max(1, keepdims=True))
        p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
    p = np.nan_to_num(p)
    rel_q, rel_p = U32 * (72 + 4 * np.minimum(d, 100)), U32 * (72 + 4 * np.minimum(np.nan_to_num(td), 100))
    g = q * rel_q
    for r in range(s.shape[0]):
        np.add.at(g[r], np.maximum(idx[r], 0) % s.shape[1], np.where((idx[r] >= 0), p[r] * rel_p[r], 0))
    lq = np.abs(np.log(np.maximum(q, 1e-300)))
    at = np.take_along_axis(lq, np.maximum(idx, 0) % s.shape[1], 1)
    loss = (p * U32 * (144 + 16 * (at + np.abs(np.log(np.maximum(p, 1e-300)))) + 8 * np.minimum(np.nan_to_num(td), 100))).sum(1)
    return loss * np.abs(w) * T * T, g * np.abs(w)[:, None] * T


VOCABS = [1, 2, 7, 100, 1000, 1023, 1025, 2047, 4000, 4096, 8190, 16385, 32001, 33000, 65535, 66000, 132000]


@pytest.mark.parametrize("place", PLACES, ids=["tight", "gaps", "odd_rows", "odd_start"])
@pytest.mark.parametrize("dt", TYPES)
def test_distillation_loss_and_gradient(dt, place):
    rng = np.random.default_rng(30)
    for V in VOCABS if place in ((0, 0), (3, 0)) else VOCABS[1::4]:
        R, k = (5, min(V, 40)) if V > 2000 else (30, min(V, 17))
        T = float(rng.choice([1.0, 2.0, 4.0, 0.7]))
        T32 = float(np.float32(T))
        say("distill", dt, place, R, V, k, T)
        s = rounded(rng.standard_normal((R, V)) * 3, dt)
        teacher = s + rng.standard_normal((R, V))
        idx = np.argsort(-teacher, 1, kind="stable")[:, :k].astype(np.int32)
        val = np.take_along_axis(teacher, idx, 1).astype(np.float32).astype(np.float64)
        w = rng.random(R).astype(np.float32).astype(np.float64) + 0.1
        if R > 4:
            idx[1, k // 2:] = -1
            idx[2, :] = -1
            idx[3, 0] = V if k > 1 else idx[3, 0]                      # not there either
            w[4] = 0.0
        loss, grad, stats, ms, i, v = _distill(s, idx, val, dt, T, w, *place)
        clean = np.where(idx >= V, -1, idx)
        want_loss, want_grad = D.distill(s, clean, val, T32, w)
        bl, bg = _distill_bounds(s, clean, val, T32, w)
        assert (np.abs(loss - want_loss) <= bl + 8 * U32 * np.abs(want_loss)).all(), (dt, V, np.abs(loss - want_loss).max())
        _close(grad, want_grad, dt, bg + 8 * U32 * np.abs(want_grad))
        if R > 4:
            assert loss[2] == 0 and loss[4] == 0 and not grad[2].any() and not grad[4].any()
        # the gradient alone, from the statistics of a call with other weights
        _, _, stats, _, _, _ = _distill(s, idx, val, dt, T, None, *place, what=("stats",))
        mg = empty(R, V, dt, *place)
        pc.distill_grad(ms, i, v, stats, mg, CODE[dt], R, V, k, T, weight=vec(w), ldl=ms.ld, ldg=mg.ld, stream=stream())
        assert mg.get().tobytes() == grad.tobytes()
        # in place
        pc.distill(ms, i, v, CODE[dt], R, V, k, T, weight=vec(w), grad=ms, ldl=ms.ld, ldg=ms.ld, stream=stream())
        assert ms.get().tobytes() == grad.tobytes()
        # logits and gradient at other alignments than each other
        again, other = _distill(s, idx, val, dt, T, w, place[0], place[1], place[0] + 5, 3)[:2]
        assert again.tobytes() == loss.tobytes() and other.tobytes() == grad.tobytes()


def test_distillation_with_an_index_that_comes_twice_and_long_lists():
    rng = np.random.default_rng(31)
    R, V, k = 6, 500, 1024
    s = rng.standard_normal((R, V)).astype(np.float32).astype(np.float64)
    idx = rng.integers(-20, V + 20, (R, k)).astype(np.int32)
    idx[0] = 7
    val = rng.standard_normal((R, k)).astype(np.float32).astype(np.float64)
    clean = np.where(idx >= V, -1, idx)
    loss, grad = _distill(s, idx, val, "f32", 2.0)[:2]
    want_loss, want_grad = D.distill(s, clean, val, 2.0)
    bl, bg = _distill_bounds(s, clean, val, 2.0, np.ones(R))
    assert (np.abs(loss - want_loss) <= bl).all()
    assert (np.abs(grad - want_grad) <= bg + 1024 * U32 * np.abs(want_grad)).all()


@pytest.mark.parametrize("V", [300, 5000, 140000])
def test_distillation_of_extreme_logits(V):
    rng = np.random.default_rng(32)
    inf, nan = np.inf, np.nan
    s = rng.standard_normal((9, V)).astype(np.float32).astype(np.float64)
    idx = np.tile(np.array([3, 8, V - 1], np.int32), (9, 1))
    val = rng.standard_normal((9, 3)).astype(np.float32).astype(np.float64)
    s[0, 50:200] = -inf                     # masked: q = 0
    s[1, 8] = -inf                          # masked where the teacher has weight: the loss is infinite, the gradient not
    s[2, 100] = nan
    s[3, 100] = inf
    s[4, :] = -inf
    val[5, 1] = -inf                        # a probability of 0
    val[6, :] = -inf                        # no probability at all: left out
    val[7, 0] = nan
    s[8, 8], val[8, 1] = -inf, -inf         # 0 * log 0
    s[6, :] = nan
    loss, grad = _distill(s, idx, val, "f32", 1.0)[:2]
    with np.errstate(all="ignore"):
        want_loss, want_grad = D.distill(s, idx, val, 1.0)
    assert loss[1] == inf and np.isnan(loss[[2, 3, 4, 7]]).all() and loss[6] == 0
    for r in (2, 3, 4, 7):
        assert np.isnan(grad[r]).all()
    assert not grad[6].any()
    for r in (0, 1, 5, 8):
        assert np.allclose(grad[r], want_grad[r], rtol=1e-5, atol=1e-7)
    for r in (0, 5, 8):
        assert loss[r] == pytest.approx(want_loss[r], rel=1e-5)
    huge = s[5:6] * 1e30                    # far apart: one logit has everything
    loss, grad = _distill(huge, idx[5:6], val[5:6], "f32", 1.0)[:2]
    with np.errstate(all="ignore"):
        want = D.distill(huge, idx[5:6], val[5:6], 1.0)
    assert np.allclose(loss, want[0], rtol=1e-5) and np.allclose(grad, want[1], rtol=1e-5, atol=1e-7)
    all_nan_but_minus = np.array([[nan, -inf, -inf]])
    loss, grad = _distill(s[5:6], idx[5:6], all_nan_but_minus, "f32", 1.0)[:2]
    assert np.isnan(loss).all() and np.isnan(grad).all()


def test_distillation_takes_the_teachers_logits_by_their_differences():
    """A teacher's logits with a large one in common (whole numbers of quarters, so that the sums are exact) are the same teacher, and
    entries that are all the type's lowest value are alike, not absent."""
    rng = np.random.default_rng(33)
    R, V, k, T = 7, 333, 20, float(np.float32(0.3))
    s = rng.standard_normal((R, V)).astype(np.float32).astype(np.float64)
    idx = np.stack([rng.permutation(V)[:k] for _ in range(R)]).astype(np.int32)
    val = rng.integers(-8, 9, (R, k)) / 4.0
    near = _distill(s, idx, val, "f32", T)
    want_loss, want_grad = D.distill(s, idx, val, T)
    bl, bg = _distill_bounds(s, idx, val, T, np.ones(R))
    for far in (2.0 ** 20, -2.0 ** 20):
        loss, grad = _distill(s, idx, val + far, "f32", T)[:2]
        assert (np.abs(loss - want_loss) <= bl).all() and (np.abs(grad - want_grad) <= bg).all()
        assert loss.tobytes() == near[0].tobytes() and grad.tobytes() == near[1].tobytes()
    lowest = np.full((R, k), float(np.finfo(np.float32).min))
    loss, grad = _distill(s, idx, lowest, "f32", T)[:2]
    same_loss, same_grad = _distill(s, idx, np.zeros((R, k)), "f32", T)[:2]
    assert loss.any() and loss.tobytes() == same_loss.tobytes() and grad.tobytes() == same_grad.tobytes()
    lowest[:, 3] = 1.0                      # one entry has everything
    loss, grad = _distill(s, idx, lowest, "f32", T)[:2]
    alone = np.full((R, k), -np.inf)
    alone[:, 3] = 1.0
    same_loss, same_grad = _distill(s, idx, alone, "f32", T)[:2]
    assert loss.tobytes() == same_loss.tobytes() and grad.tobytes() == same_grad.tobytes()


def test_distillation_at_temperatures_whose_square_or_quotients_pass_32_bits():
    """Logits of whole 2^-10, whose differences are exact.  Cold: one entry has everything (p = q = 1 at their largest), so that the loss is T
    times what the network's logit there is short of its largest, one product, and the gradient -T and T.  Hot: all exponentials are 1, so
    that the loss is T^2 * log(V / k), the difference of two logarithms of two units of at most 2 log(V), and two products."""
    rng = np.random.default_rng(35)
    R, V, k = 5, 200, 7
    s = rng.permuted(np.arange(V) / 1024.0 * np.ones((R, 1)), axis=1)
    idx = np.stack([rng.permutation(V)[:k] for _ in range(R)]).astype(np.int32)
    val = rng.permuted(np.arange(k) / 4.0 * np.ones((R, 1)), axis=1)
    best = np.take_along_axis(idx, val.argmax(1)[:, None], 1)[:, 0]
    short = s.max(1) - s[np.arange(R), best]
    for T in (1e-20, 1e-25, 1e-30):
        T32 = float(np.float32(T))
        loss, grad = _distill(s, idx, val, "f32", T)[:2]
        assert (np.abs(loss - T32 * short) <= 2 * U32 * T32 * short).all(), T
        want = np.zeros((R, V))
        want[np.arange(R), s.argmax(1)] += T32
        want[np.arange(R), best] -= T32
        assert (np.abs(grad - want) <= 8 * U32 * T32).all(), T
    for T, V2, k2 in ((2e19, 4, 2), (1e19, 300, 40), (1.8e19, 3, 3), (1e25, 1, 1), (3e38, 1, 1), (1e19, 2, 2)):
        T32 = float(np.float32(T))
        loss, grad = _distill(s[:, :V2], np.arange(k2)[None, :].repeat(R, 0), val[:, :1].repeat(k2, 1), "f32", T)[:2] if V2 <= V else \
            _distill(np.zeros((R, V2)), np.arange(k2)[None, :].repeat(R, 0), np.zeros((R, k2)), "f32", T)[:2]
        want = T32 * T32 * np.log(V2 / k2)
        assert (np.abs(loss - want) <= T32 * T32 * 8 * U32 * 2 * np.log(V2)).all(), (T, V2, k2, loss, want)
        assert np.isfinite(grad).all()


def test_small_probabilities_are_as_exact_as_large_ones_in_32_bits():
    """Logits of whole 2^-10, whose differences are exact, down to 60 T below the largest.  In units of 2^-24: the sum of 400 exponentials
    in 14 additions on top of each other 14, its exponentials 4, the element's exponential 4, two products and two quotients 4: 26, with
    the second-order terms 28."""
    rng = np.random.default_rng(34)
    R, V, T = 8, 400, 0.25
    s = -rng.integers(0, 15 * 1024, (R, V)) / 1024.0
    s[:, 17] = 0.0
    _, grad = _distill(s, np.full((R, 1), 17, np.int32), np.zeros((R, 1)), "f32", T)[:2]
    q = np.exp(s / T)
    q /= q.sum(1, keepdims=True)
    others = np.arange(V) != 17
    assert (np.abs(grad[:, others] - T * q[:, others]) <= 28 * U32 * T * q[:, others]).all()


def test_distillation_of_more_rows_than_a_launch_takes():
    """2^26 rows of 64 threads are as many threads as no launch has."""
    import torch
    R, T = (1 << 26) + 5, 2.0
    g = torch.Generator(device="cuda").manual_seed(5)
    s = torch.randn(R, 2, generator=g, device="cuda").half()
    idx = torch.randint(0, 2, (R, 1), generator=g, device="cuda", dtype=torch.int32)
    val = torch.zeros(R, 1, device="cuda")
    loss, grad, stats = torch.full((R,), 55.0, device="cuda"), torch.full_like(s, 55.0), torch.full((R, 2), 55.0, device="cuda")
    say("distill", R)
    pc.distill(s, idx, val, pc.F16, R, 2, 1, T, loss=loss, grad=grad, stats=stats, stream=stream())
    again = torch.full_like(grad, 55.0)
    pc.distill_grad(s, idx, val, stats, again, pc.F16, R, 2, 1, T, stream=stream())
    torch.cuda.synchronize()
    assert bool((again == grad).all())
    for at in range(0, R, 1 << 24):
        part = slice(at, at + (1 << 24))
        x, i = s[part].double(), idx[part].long()
        far = (x.gather(1, 1 - i) - x.gather(1, i))[:, 0] / T       # the other logit's distance: log q = -log(1 + exp(far))
        want = T * T * torch.log1p(torch.exp(far))
        # (the largest logit's own exponential is 1: the loss is off by units of log(norm) and of the distance, 6 units of 1 + |far| each)
        assert bool(((loss[part].double() - want).abs() <= T * T * 12 * U32 * (1 + far.abs())).all())
        q = 1 / (1 + torch.exp(far))
        own, other = grad[part].double().gather(1, i)[:, 0], grad[part].double().gather(1, 1 - i)[:, 0]
        for have, right in ((own, T * (q - 1)), (other, T * (1 - q))):
            # half a step of fp16, and 16 units of 32 bits of the terms, T at most
            assert bool(((have - right).abs() <= HALF["f16"] * right.abs() + TINY["f16"] + 16 * U32 * T * (1 + far.abs())).all())


def test_elementwise_passes_of_more_pieces_than_a_launch_takes():
    """Rows of one element, 2^28 to a launch, and a weight gradient of more floats than that."""
    import torch
    M = (1 << 28) + 3
    z = torch.ones(M, dtype=torch.bfloat16, device="cuda")
    z[1::2] = -1
    dz = torch.full_like(z, 3.0)
    say("activation_grad", M)
    pc.activation_grad(dz, z, dz, pc.BF16, M, 1, pc.ACT_RELU, stream=stream())
    torch.cuda.synchronize()
    assert bool((dz[0::2] == 3).all()) and not bool(dz[1::2].any())
    del z, dz
    N, K = (1 << 14) + 1, 1 << 14
    dw, db = torch.full((N * K + 64,), 55.0, device="cuda"), torch.full((N + 64,), 55.0, device="cuda")
    say("grad_weight of no rows", N, K)
    pc.linear_grad_weight(None, None, dw, pc.F16, 0, N, K, db=db, stream=stream())
    torch.cuda.synchronize()
    assert not bool(dw[:N * K].any()) and bool((dw[N * K:] == 55).all()) and not bool(db[:N].any()) and bool((db[N:] == 55).all())


# ------------------------------------------------------------------------------------------------------------------ together

def _head_step(t, dt, st, scratch):
    """Norm, two linear layers with a residual, distillation, and all the way back, on stream st."""
    M, C, H, V, k = t["M"], t["C"], t["H"], t["V"], t["k"]
    c = CODE[dt]
    pc.layer_norm(t["x"], t["n"], c, M, C, gamma=t["gamma"], beta=t["beta"], mean=t["mean"], rstd=t["rstd"], stream=st)
    pc.linear(t["n"], t["w1"], t["h"], c, M, H, C, bias=t["b1"], z=t["z"], act=pc.ACT_GELU_TANH, stream=st, **scratch[0].args())
    pc.linear(t["h"], t["w2"], t["l"], c, M, V, H, bias=t["b2"], stream=st, **scratch[1].args())
    pc.distill(t["l"], t["i"], t["v"], c, M, V, k, 2.0, weight=t["weight"], loss=t["loss"], grad=t["dl"], stream=st)
    pc.linear_grad_input(t["dl"], t["w2"], t["dz"], c, M, V, H, z=t["z"], act=pc.ACT_GELU_TANH, stream=st, **scratch[2].args())
    pc.linear_grad_weight(t["dl"], t["h"], t["dw2"], c, M, V, H, db=t["db2"], stream=st, **scratch[3].args())
    pc.linear_grad_input(t["dz"], t["w1"], t["dn"], c, M, H, C, stream=st, **scratch[4].args())
    pc.linear_grad_weight(t["dz"], t["n"], t["dw1"], c, M, H, C, db=t["db1"], stream=st, **scratch[5].args())
    pc.layer_norm_grad(t["dn"], t["x"], t["dx"], t["mean"], t["rstd"], c, M, C, gamma=t["gamma"], dgamma=t["dgamma"], dbeta=t["dbeta"],
                       stream=st, **scratch[6].args())


def _head(dt, seed):
    import torch
    M, C, H, V, k = 70, 96, 200, 333, 9
    rng = np.random.default_rng(seed)
    a = {"x": rng.standard_normal((M, C)), "w1": rng.standard_normal((H, C)) / 10, "w2": rng.standard_normal((V, H)) / 6}
    a = {n: rounded(v, dt) for n, v in a.items()}
    f = {"gamma": rng.standard_normal(C), "beta": rng.standard_normal(C), "b1": rng.standard_normal(H), "b2": rng.standard_normal(V),
         "weight": rng.random(M) / M}
    f = {n: v.astype(np.float32) for n, v in f.items()}
    f["weight"][5] = 0
    i = np.stack([rng.permutation(V)[:k] for _ in range(M)]).astype(np.int32)
    v = (rng.standard_normal((M, k)) * 2).astype(np.float32)
    t = {"M": M, "C": C, "H": H, "V": V, "k": k, "i": torch.from_numpy(i).cuda(), "v": torch.from_numpy(v).cuda()}
    t.update({n: Mat(x, dt) for n, x in a.items()})
    t.update({n: vec(x) for n, x in f.items()})
    for n, cols in (("n", C), ("h", H), ("z", H), ("l", V), ("dl", V), ("dz", H), ("dn", C), ("dx", C)):
        t[n] = empty(M, cols, dt)
    for n, shape in (("mean", (1, M)), ("rstd", (1, M)), ("loss", (1, M)), ("dw1", (H, C)), ("dw2", (V, H)), ("db1", (1, H)), ("db2", (1, V)),
                     ("dgamma", (1, C)), ("dbeta", (1, C))):
        t[n] = empty(*shape, "f32")
    c = CODE[dt]
    scratch = [Scratch(n) for n in (pc.linear_workspace(c, M, H, C), pc.linear_workspace(c, M, V, H), pc.linear_grad_input_workspace(c, M, V, H),
                                    pc.linear_grad_weight_workspace(c, M, V, H), pc.linear_grad_input_workspace(c, M, H, C),
                                    pc.linear_grad_weight_workspace(c, M, H, C), pc.layer_norm_grad_workspace(c, M, C))]
    return t, scratch, a, f, i, v


OUT = ("loss", "dx", "dw1", "dw2", "db1", "db2", "dgamma", "dbeta")


@pytest.mark.parametrize("dt", TYPES)
def test_a_head_is_trained_one_step(dt):
    """All operators in a row against the float64 forms.  The tensors between them are stored in dt: an error of half a step each, of which
    six follow each other, so that a gradient may be off by some six half steps of its norm; twice that is allowed (fp32: 1e-5)."""
    t, scratch, a, f, i, v = _head(dt, 40)
    _head_step(t, dt, stream(), scratch)
    n, _, _ = D.layer_norm(a["x"], f["gamma"], f["beta"])
    h, z = D.linear(n, a["w1"], f["b1"], name="gelu_tanh")
    l, _ = D.linear(h, a["w2"], f["b2"])
    loss, dl = D.distill(l, i, v.astype(np.float64), 2.0, f["weight"])
    dz = D.linear_grad_input(dl, a["w2"], z, "gelu_tanh")
    dw2, db2 = D.linear_grad_weight(dl, h)
    dn = D.linear_grad_input(dz, a["w1"])
    dw1, db1 = D.linear_grad_weight(dz, n)
    dx, dgamma, dbeta = D.layer_norm_grad(dn, a["x"], f["gamma"])
    want = dict(loss=loss, dx=dx, dw1=dw1, dw2=dw2, db1=db1, db2=db2, dgamma=dgamma, dbeta=dbeta)
    for name in OUT:
        got = t[name].get()
        got = got[0] if want[name].ndim == 1 else got
        off = np.linalg.norm(got - want[name]) / np.linalg.norm(want[name])
        assert off <= (1e-5 if dt == "f32" else 12 * HALF[dt]), (name, off)


def test_a_head_on_another_stream_and_in_graphs():
    """The same step eagerly, on a stream of its own, and as two captured graphs with workspaces of their own that are replayed in turn,
    with eager work and synchronizations between the replays: bit for bit the same."""
    import torch
    t, scratch, *_ = _head("bf16", 41)
    _head_step(t, "bf16", stream(), scratch)
    want = {n: t[n].get().tobytes() for n in OUT}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for n in OUT:
        t[n].view.fill_(5.0)
    torch.cuda.synchronize()
    _head_step(t, "bf16", side.cuda_stream, scratch)
    torch.cuda.synchronize()
    assert {n: t[n].get().tobytes() for n in OUT} == want
    graphs = []
    for _ in range(2):
        t2, s2, *_ = _head("bf16", 41)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            _head_step(t2, "bf16", torch.cuda.current_stream().cuda_stream, s2)
        graphs.append((g, t2, s2))
    for turn in range(3):
        for g, t2, s2 in graphs:
            for n in OUT:
                t2[n].view.fill_(float(turn))
            for s in s2:
                s.buf[:s.n] = 0xFF
            torch.cuda.synchronize()
            g.replay()
        _head_step(t, "bf16", stream(), scratch)
        torch.cuda.synchronize()
        for _, t2, _ in graphs:
            assert {n: t2[n].get().tobytes() for n in OUT} == want, turn
        assert {n: t[n].get().tobytes() for n in OUT} == want


def test_behind_a_pruned_layer():
    """The dense operators next to the pruned ones: a channel-minor pruned 3x3 layer, the norm over its channels, a dense 1x1 layer with the
    residual of the map, ReLU behind it; and the pruned 3x3 layer's output gradient from their backward pass."""
    import torch
    from workloads import layers as L
    from gpu_util import GpuLayer
    spec = L.LayerSpec(cfg=31, idx=0, name="head", N=2, C=32, F=64, H=12, W=10, stride=1, pad=1, dtype="f16", K=8, keep=1.0)
    layer = GpuLayer(spec, use_bias=True)
    x = L.gen_activations(spec)
    xh = torch.from_numpy(x).cuda().permute(0, 2, 3, 1).contiguous()
    M, C, N = 2 * 12 * 10, 64, 64
    y = torch.empty((M, C), dtype=torch.float16, device="cuda")
    pc.conv3x3(xh, y, layer.packed, layer.d_bias, 2, 12, 10, 1, 1, pc.FLAG_RELU | pc.FLAG_NHWC, stream())
    n, o = torch.empty_like(y), torch.empty_like(y)
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    pc.layer_norm(y, n, pc.F16, M, C, mean=mean, rstd=rstd, stream=stream())
    rng = np.random.default_rng(42)
    w = rounded(rng.standard_normal((N, C)) / 8, "f16")
    dw = torch.from_numpy(w).cuda().half()
    ws = Scratch(pc.linear_workspace(pc.F16, M, N, C))
    pc.linear(n, dw, o, pc.F16, M, N, C, residual=y, act=pc.ACT_RELU, flags=pc.FLAG_RESIDUAL_FIRST, stream=stream(), **ws.args())
    g = rounded(rng.standard_normal((M, N)), "f16")
    dg = torch.from_numpy(g).cuda().half()
    dz, dn, dy = torch.empty_like(o), torch.empty_like(o), torch.empty_like(o)
    pc.activation_grad(dg, o, dz, pc.F16, M, N, pc.ACT_RELU, stream=stream())            # (o stands for z: ReLU)
    ws2 = Scratch(pc.linear_grad_input_workspace(pc.F16, M, N, C))
    pc.linear_grad_input(dz, dw, dn, pc.F16, M, N, C, stream=stream(), **ws2.args())
    pc.layer_norm_grad(dn, y, dy, mean, rstd, pc.F16, M, C, stream=stream())
    torch.cuda.synchronize()
    hy = layer.oracle(x, relu=True).transpose(0, 2, 3, 1).reshape(M, C)
    hn = D.layer_norm(hy)[0]
    ho, hz = D.linear(hn, w, None, hy, "relu", True)
    off = np.linalg.norm(o.double().cpu().numpy() - ho) / np.linalg.norm(ho)
    assert off <= 6 * HALF["f16"], off                     # three stored tensors in a row
    sure = np.abs(hz) > 0.02                               # (where z is near 0 the stored one may have the other sign)
    hd = np.where(sure, g * D.act_slope(hz, "relu"), dz.double().cpu().numpy())
    assert np.array_equal(dz.double().cpu().numpy(), hd)
    want = D.layer_norm_grad(D.linear_grad_input(hd, w), hy)[0]
    off = np.linalg.norm(dy.double().cpu().numpy() - want) / np.linalg.norm(want)
    assert off <= 12 * HALF["f16"], off
    layer.free()


def test_offsets_that_pass_32_bits():
    """Rows behind the first 4 GiB of a tensor: the last rows equal the same rows alone."""
    import torch
    D_, rows = 4096, (1 << 20) + 70000                     # 2.2e9 .. bytes: 1,118,576 x 4096 bf16 = 9.2 GB
    x = torch.empty((rows, D_), dtype=torch.bfloat16, device="cuda")
    torch.manual_seed(3)
    block = torch.randn((4096, D_), device="cuda").bfloat16()
    for at in range(0, rows, 4096):
        x[at:at + 4096] = block[:min(4096, rows - at)]
    x[rows - 300:] = torch.randn((300, D_), device="cuda").bfloat16()
    y = torch.empty_like(x)
    tail, small = x[rows - 300:].contiguous(), torch.empty((300, D_), dtype=torch.bfloat16, device="cuda")
    pc.layer_norm(x, y, pc.BF16, rows, D_, stream=stream())
    pc.layer_norm(tail, small, pc.BF16, 300, D_, stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(y[rows - 300:], small)
    # a product over the same rows: its last rows, and the input gradient of all of them
    N = 64
    w = torch.randn((N, D_), device="cuda").bfloat16()
    out = torch.zeros((rows, N), dtype=torch.bfloat16, device="cuda")
    assert pc.linear_workspace(pc.BF16, rows, N, D_) == 0
    pc.linear(x, w, out, pc.BF16, rows, N, D_, stream=stream())
    torch.cuda.synchronize()
    want = (tail.double() @ w.double().t())
    size = torch.sqrt((tail.double() ** 2) @ (w.double() ** 2).t())
    assert bool(((out[rows - 300:].double() - want).abs() <= HALF["bf16"] * want.abs() + 6 * U32 * 64 * size).all())
    pc.linear_grad_input(out, w, y, pc.BF16, rows, N, D_, stream=stream())
    torch.cuda.synchronize()
    want = out[rows - 300:].double() @ w.double()
    size = torch.sqrt((out[rows - 300:].double() ** 2) @ (w.double() ** 2))
    assert bool(((y[rows - 300:].double() - want).abs() <= HALF["bf16"] * want.abs() + 6 * U32 * 8 * size).all())
    # and the weight gradient over all rows: whole numbers in the last rows alone
    out.zero_()
    out[rows - 5:] = 1.0
    dw = torch.empty((N, D_), device="cuda")
    ws = Scratch(pc.linear_grad_weight_workspace(pc.BF16, rows, N, D_))
    pc.linear_grad_weight(out, x, dw, pc.BF16, rows, N, D_, stream=stream(), **ws.args())
    torch.cuda.synchronize()
    want = x[rows - 5:].double().sum(0)
    assert bool(((dw.double() - want).abs() <= 8 * U32 * x[rows - 5:].double().abs().sum(0)).all())


@pytest.mark.parametrize("dt", TYPES)
def test_in_place_in_every_path(dt):
    """A residual that is y, an added gradient that is dx, a norm's y that is x, its dx that is x or dy: the bits of the call beside them."""
    import torch
    rng = np.random.default_rng(44)
    real = lambda *shape: torch.from_numpy(rng.standard_normal(shape)).cuda().to(ttype(dt))  # noqa: E731
    for M, N, K, pad in [(3, 70, 5000, 0), (150, 140, 203, 0), (100, 130, 5000, 0), (1030, 1100, 136, 0), (2100, 2200, 264, 5), (4600, 6143, 72, 0)]:
        say("in place", dt, M, N, K, pad)
        x, w, r = real(M, K + pad), real(N, K + pad), real(M, N)
        ws = Scratch(max(pc.linear_workspace(CODE[dt], M, N, K), pc.linear_grad_input_workspace(CODE[dt], M, N, K)))
        for flags in (0, pc.FLAG_RESIDUAL_FIRST):
            y, z, one = r.clone(), torch.empty_like(r), torch.empty_like(r)
            for out in (one, y):
                pc.linear(x, w, out, CODE[dt], M, N, K, residual=r if out is one else y, z=z, act=pc.ACT_SILU, flags=flags, ldx=K + pad,
                          ldw=K + pad, stream=stream(), **ws.args())
            assert torch.equal(y, one), (dt, M, N, K, flags)
        add = real(M, K)
        dx, one = add.clone(), torch.empty_like(add)
        for out in (one, dx):
            pc.linear_grad_input(r, w, out, CODE[dt], M, N, K, z=x, act=pc.ACT_SILU, add=add if out is one else dx, ldw=K + pad, ldz=K + pad,
                                 stream=stream(), **ws.args())
        assert torch.equal(dx, one), (dt, M, N, K)
    for Dn in (33, 100, 200, 500, 1000, 2000, 4001, 8000, 16001, 33000):
        rows = max(7, 2000000 // Dn // 8)
        say("norm in place", dt, rows, Dn)
        x, dy, gamma = real(rows, Dn), real(rows, Dn), vec(rng.standard_normal(Dn))
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        one, same = torch.empty_like(x), x.clone()
        for a, b in ((x, one), (same, same)):
            pc.layer_norm(a, b, CODE[dt], rows, Dn, gamma=gamma, beta=gamma, mean=mean, rstd=rstd, stream=stream())
        assert torch.equal(one, same), (dt, rows, Dn)
        need, got = pc.layer_norm_grad_workspace(CODE[dt], rows, Dn), []
        for which in range(3):
            a, g = x.clone(), dy.clone()
            out = (torch.empty_like(x), a, g)[which]
            sums, ws = torch.empty(2, Dn, device="cuda"), Scratch(need)
            pc.layer_norm_grad(g, a, out, mean, rstd, CODE[dt], rows, Dn, gamma=gamma, dgamma=sums[0], dbeta=sums[1], stream=stream(), **ws.args())
            got.append((out, sums))
        assert all(torch.equal(o, got[0][0]) and torch.equal(s, got[0][1]) for o, s in got[1:]), (dt, rows, Dn)


def test_as_many_rows_as_there_may_be():
    """2^30 rows of products and 2^31 - 1 of a norm, a block of rows over and over: every copy of it gives what the block alone gives."""
    import torch
    rng = np.random.default_rng(43)
    copies, rows, K, N = 1 << 10, 1 << 20, 8, 16
    M = copies * rows
    block, w = (torch.from_numpy(whole(rng, s, 3)).cuda().bfloat16() for s in ((rows, K), (N, K)))
    x = torch.empty((copies, rows, K), dtype=torch.bfloat16, device="cuda")
    x.copy_(block)
    y = torch.empty((copies, rows, N), dtype=torch.bfloat16, device="cuda")
    assert pc.linear_workspace(pc.BF16, M, N, K) == 0 and pc.linear_grad_input_workspace(pc.BF16, M, N, K) == 0
    say("linear", M)
    pc.linear(x, w, y, pc.BF16, M, N, K, act=pc.ACT_RELU, stream=stream())
    torch.cuda.synchronize()
    want = (block.float() @ w.float().t()).clamp(min=0).bfloat16()           # (whole numbers below 72)
    assert bool((y[0] == want).all()) and all(bool((y[at:at + 64] == y[0]).all()) for at in range(0, copies, 64))
    say("linear_grad_input", M)
    pc.linear_grad_input(y, w, x, pc.BF16, M, N, K, stream=stream())
    torch.cuda.synchronize()
    want = (want.float() @ w.float()).bfloat16()
    assert bool((x[0] == want).all()) and all(bool((x[at:at + 64] == x[0]).all()) for at in range(0, copies, 64))
    y[:-1] = 0                                                               # the last block's rows alone
    y[-1, :-9] = 0
    x.copy_(block)
    dw = torch.full((N, K), 55.0, device="cuda")
    ws = Scratch(pc.linear_grad_weight_workspace(pc.BF16, M, N, K))
    say("linear_grad_weight", M)
    pc.linear_grad_weight(y, x, dw, pc.BF16, M, N, K, stream=stream(), **ws.args())
    torch.cuda.synchronize()
    ws.check()
    assert bool((dw.double() == y[-1, -9:].double().t() @ block[-9:].double()).all())
    del x, y
    M, D_ = (1 << 31) - 1, 2
    x = torch.empty((1 << 31, D_), dtype=torch.bfloat16, device="cuda")
    x.view(1 << 10, 1 << 21, D_).copy_(torch.randn((1 << 21, D_), device="cuda"))
    small, last = torch.empty((1 << 21, D_), dtype=torch.bfloat16, device="cuda"), x[-1].clone()
    pc.layer_norm(x, small, pc.BF16, 1 << 21, D_, stream=stream())
    say("layer_norm", M)
    pc.layer_norm(x, x, pc.BF16, M, D_, stream=stream())
    torch.cuda.synchronize()
    assert bool((x[-1] == last).all())
    x[-1] = small[-1]
    assert all(bool((x.view(1 << 10, 1 << 21, D_)[at:at + 64] == small).all()) for at in range(0, 1 << 10, 64))
