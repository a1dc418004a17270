"""What the entries of include/pconv_dense.h refuse, and what they ask for; the checks come before any launch, so no GPU is needed."""
import ctypes

import pytest

import paper_2001_07710_amd as pc


class P:
    """A pointer that is never followed."""

    def __init__(self, at=1 << 20):
        self.at = at

    def data_ptr(self):
        return self.at


X, W, Y, Z, R, B, WS = (P((i + 1) << 20) for i in range(7))
BIG = 1 << 40


def code(f, *a, **k):
    pc.ensure_built()
    with pytest.raises(pc.PconvError) as e:
        f(*a, **k)
    return e.value.code


@pytest.mark.parametrize("dtype", [pc.F32, pc.F16, pc.BF16])
def test_linear_refuses(dtype):
    ok = dict(bias=B, residual=R, z=Z, workspace=WS, workspace_bytes=BIG)
    c = lambda *a, **k: code(pc.linear, *a, **{**ok, **k})  # noqa: E731
    assert c(X, W, Y, 3, 4, 5, 6) == pc.EINVAL and c(X, W, Y, -1, 4, 5, 6) == pc.EINVAL
    assert c(X, W, Y, dtype, -1, 5, 6) == pc.ESHAPE and c(X, W, Y, dtype, 4, 0, 6) == pc.ESHAPE and c(X, W, Y, dtype, 4, 5, 0) == pc.ESHAPE
    assert c(X, W, Y, dtype, 4, 5, 6, act=5) == pc.EINVAL and c(X, W, Y, dtype, 4, 5, 6, act=-1) == pc.EINVAL
    assert c(X, W, Y, dtype, 4, 5, 6, flags=1) == pc.EINVAL and c(X, W, Y, dtype, 4, 5, 6, flags=16) == pc.EINVAL
    for k in ("ldx", "ldw", "ldr", "ldy"):
        assert c(X, W, Y, dtype, 4, 5, 6, **{k: 4}) == pc.ESHAPE
        assert c(X, W, Y, dtype, 4, 5, 6, **{k: -8}) == pc.ESHAPE
        assert c(X, W, Y, dtype, 4, 5, 6, **{k: (1 << 20) + 1}) == pc.EUNSUPPORTED
    assert c(X, W, Y, dtype, 4, 5, (1 << 20) + 1) == pc.EUNSUPPORTED
    assert c(None, W, Y, dtype, 4, 5, 6) == pc.EINVAL and c(X, None, Y, dtype, 4, 5, 6) == pc.EINVAL
    assert c(X, W, None, dtype, 4, 5, 6) == pc.EINVAL
    odd = P((1 << 20) + 1)
    for a in ((odd, W, Y), (X, odd, Y), (X, W, odd)):
        assert c(*a, dtype, 4, 5, 6) == pc.EINVAL
    for k in ("bias", "residual", "z"):
        assert c(X, W, Y, dtype, 4, 5, 6, **{k: odd}) == pc.EINVAL
    assert c(X, W, Y, dtype, 4, 5, 6, bias=P((1 << 20) + 2)) == pc.EINVAL
    need = pc.linear_workspace(dtype, 48, 64, 20000)
    assert need > 0
    assert c(X, W, Y, dtype, 48, 64, 20000, workspace=None) == pc.EINVAL
    assert c(X, W, Y, dtype, 48, 64, 20000, workspace_bytes=need - 1) == pc.EINVAL
    assert c(X, W, Y, dtype, 48, 64, 20000, workspace=P((1 << 20) + 8)) == pc.EINVAL
    pc.linear(None, None, None, dtype, 0, 5, 6)                       # no rows: nothing to do


@pytest.mark.parametrize("dtype", [pc.F32, pc.F16, pc.BF16])
def test_linear_gradients_refuse(dtype):
    ok = dict(workspace=WS, workspace_bytes=BIG)
    c = lambda *a, **k: code(pc.linear_grad_input, *a, **{**ok, **k})  # noqa: E731
    assert c(X, W, Y, 7, 4, 5, 6) == pc.EINVAL and c(X, W, Y, dtype, 4, 0, 6) == pc.ESHAPE
    assert c(X, W, Y, dtype, 4, 5, 6, act=pc.ACT_RELU) == pc.EINVAL              # no z
    assert c(X, W, Y, dtype, 4, 5, 6, act=9, z=Z) == pc.EINVAL
    for k in ("lddz", "ldw", "ldz", "lda", "lddx"):
        assert c(X, W, Y, dtype, 4, 7, 6, z=Z, add=R, act=pc.ACT_SILU, **{k: 5}) == pc.ESHAPE
        assert c(X, W, Y, dtype, 4, 7, 6, z=Z, add=R, act=pc.ACT_SILU, **{k: 1 << 21}) == pc.EUNSUPPORTED
    for a in ((None, W, Y), (X, None, Y), (X, W, None)):
        assert c(*a, dtype, 4, 5, 6) == pc.EINVAL
    need = pc.linear_grad_input_workspace(dtype, 48, 20000, 64)
    assert need > 0 and c(X, W, Y, dtype, 48, 20000, 64, workspace_bytes=need - 1) == pc.EINVAL
    pc.linear_grad_input(None, None, None, dtype, 0, 5, 6, act=pc.ACT_GELU)
    c = lambda *a, **k: code(pc.linear_grad_weight, *a, **{**ok, **k})  # noqa: E731
    assert c(X, W, Y, 7, 4, 5, 6) == pc.EINVAL and c(X, W, Y, dtype, 4, 5, -6) == pc.ESHAPE
    assert c(X, W, None, dtype, 4, 5, 6) == pc.EINVAL and c(None, W, Y, dtype, 4, 5, 6) == pc.EINVAL
    assert c(X, W, P((1 << 20) + 2), dtype, 4, 5, 6) == pc.EINVAL and c(X, W, Y, dtype, 4, 5, 6, db=P((1 << 20) + 2)) == pc.EINVAL
    assert c(X, W, Y, dtype, 4, 7, 6, lddz=5) == pc.ESHAPE and c(X, W, Y, dtype, 4, 7, 6, ldx=5) == pc.ESHAPE
    need = pc.linear_grad_weight_workspace(dtype, 20000, 48, 64)
    assert need > 0 and c(X, W, Y, dtype, 20000, 48, 64, workspace_bytes=need - 1) == pc.EINVAL
    c = lambda *a, **k: code(pc.activation_grad, *a, **k)  # noqa: E731
    assert c(X, Z, Y, dtype, 4, 5, 11) == pc.EINVAL and c(X, Z, Y, dtype, -4, 5, 1) == pc.ESHAPE
    assert c(X, None, Y, dtype, 4, 5, 1) == pc.EINVAL and c(X, Z, Y, dtype, 4, 5, 1, ldz=4) == pc.ESHAPE
    pc.activation_grad(None, None, None, dtype, 0, 5, 1)


@pytest.mark.parametrize("dtype", [pc.F32, pc.F16, pc.BF16])
def test_layer_norm_refuses(dtype):
    c = lambda *a, **k: code(pc.layer_norm, *a, **k)  # noqa: E731
    assert c(X, Y, 4, 4, 5) == pc.EINVAL and c(X, Y, dtype, -1, 5) == pc.ESHAPE and c(X, Y, dtype, 4, 0) == pc.ESHAPE
    for eps in (-1e-5, float("nan")):
        assert c(X, Y, dtype, 4, 5, eps=eps) == pc.EINVAL
    assert c(X, Y, dtype, 4, 5, ldx=4) == pc.ESHAPE and c(X, Y, dtype, 4, 5, ldy=4) == pc.ESHAPE
    assert c(X, Y, dtype, 4, (1 << 20) + 1) == pc.EUNSUPPORTED
    assert c(None, Y, dtype, 4, 5) == pc.EINVAL and c(X, None, dtype, 4, 5) == pc.EINVAL and c(X, P(3), dtype, 4, 5) == pc.EINVAL
    for k in ("gamma", "beta", "mean", "rstd"):
        assert c(X, Y, dtype, 4, 5, **{k: P(6)}) == pc.EINVAL
    pc.layer_norm(None, None, dtype, 0, 5)
    need = pc.layer_norm_grad_workspace(dtype, 5000, 64)
    ok = dict(dgamma=B, dbeta=Z, workspace=WS, workspace_bytes=need)
    c = lambda *a, **k: code(pc.layer_norm_grad, *a, **{**ok, **k})  # noqa: E731
    assert need > 0 and c(X, W, Y, R, B, dtype, 5000, 64, workspace_bytes=need - 1) == pc.EINVAL
    assert c(X, W, Y, R, B, dtype, 5000, 64, workspace=P((1 << 20) + 4)) == pc.EINVAL
    for a in ((None, W, Y, R, B), (X, None, Y, R, B), (X, W, Y, None, B), (X, W, Y, R, None), (X, W, P(5), R, B)):
        assert c(*a, dtype, 5000, 64) == pc.EINVAL
    assert c(X, W, Y, R, B, dtype, 5000, 64, lddx=63) == pc.ESHAPE and c(X, W, Y, R, B, 3, 5000, 64) == pc.EINVAL
    pc.layer_norm_grad(None, None, Y, None, None, dtype, 0, 64)
    pc.layer_norm_grad(X, W, None, R, B, dtype, 5000, 64)            # nothing is asked for


@pytest.mark.parametrize("dtype", [pc.F32, pc.F16, pc.BF16])
def test_distillation_refuses(dtype):
    ok = dict(loss=B, grad=Y)
    c = lambda *a, **k: code(pc.distill, *a, **{**ok, **k})  # noqa: E731
    assert c(X, W, Z, 5, 4, 100, 3, 1.0) == pc.EINVAL
    assert c(X, W, Z, dtype, -4, 100, 3, 1.0) == pc.ESHAPE and c(X, W, Z, dtype, 4, 0, 3, 1.0) == pc.ESHAPE
    assert c(X, W, Z, dtype, 4, 100, 0, 1.0) == pc.ESHAPE and c(X, W, Z, dtype, 4, 100, 1025, 1.0) == pc.EUNSUPPORTED
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert c(X, W, Z, dtype, 4, 100, 3, T) == pc.EINVAL
    assert c(X, W, Z, dtype, 4, 100, 3, 1.0, ldl=99) == pc.ESHAPE and c(X, W, Z, dtype, 4, 100, 3, 1.0, ldg=1 << 21) == pc.EUNSUPPORTED
    assert c(X, W, Z, dtype, 4, 100, 3, 1.0, loss=None, grad=None) == pc.EINVAL
    for a in ((None, W, Z), (X, None, Z), (X, W, None), (P(3), W, Z), (X, P(6), Z), (X, W, P(6))):
        assert c(*a, dtype, 4, 100, 3, 1.0) == pc.EINVAL
    assert c(X, W, Z, dtype, 4, 100, 3, 1.0, weight=P(6)) == pc.EINVAL and c(X, W, Z, dtype, 4, 100, 3, 1.0, stats=P(6)) == pc.EINVAL
    pc.distill(None, None, None, dtype, 0, 100, 3, 1.0, loss=B)
    c = lambda *a: code(pc.distill_grad, *a)  # noqa: E731
    assert c(X, W, Z, None, Y, dtype, 4, 100, 3, 1.0) == pc.EINVAL and c(X, W, Z, B, None, dtype, 4, 100, 3, 1.0) == pc.EINVAL
    assert c(X, W, Z, B, Y, dtype, 4, 100, 3, 0.0) == pc.EINVAL


def test_distillation_refuses_temperatures_whose_exponents_overflow():
    """The kernel takes exp(d / T) as 2^(d * log2(e) / T): log2(e) / T is finite from 1.4427 / (2^128 - 2^103) = 4.2397e-39 on."""
    for T in (1e-45, 2.9e-39, 2.95e-39, 3e-39, 4.2e-39):
        assert code(pc.distill, X, W, Z, pc.F16, 4, 100, 3, T, loss=B, grad=Y) == pc.EINVAL
        assert code(pc.distill_grad, X, W, Z, B, Y, pc.F16, 4, 100, 3, T) == pc.EINVAL
    for T in (4.25e-39, 1e-38, 1e-30, 1e30, 3.4e38):
        pc.distill(None, None, None, pc.F16, 0, 100, 3, T, loss=B)


def test_sizes_at_the_end_of_their_range():
    """Plans of the largest sizes: no overflow, a workspace of whole parts, and none where there is nothing to share."""
    pc.ensure_built()
    big = (1 << 31) - 1
    for dtype in (pc.F32, pc.F16, pc.BF16):
        assert pc.linear_workspace(dtype, 1 << 30, 1 << 20, 1) == 0
        assert pc.linear_workspace(dtype, 1 << 30, 1 << 20, 1 << 20) == 0
        for sizes in ((big, 64, 64), (64, big, 64), (64, 64, big)):
            for f in (pc.linear_workspace, pc.linear_grad_input_workspace, pc.linear_grad_weight_workspace):
                assert code(f, dtype, *sizes) == pc.EUNSUPPORTED
        assert pc.linear_grad_weight_workspace(dtype, 0, 64, 64) == 0 and pc.layer_norm_grad_workspace(dtype, 0, 64) == 0
        assert pc.linear_grad_weight_workspace(dtype, 1 << 30, 64, 64) % 16 == 0
        assert pc.layer_norm_grad_workspace(dtype, big, 64) > 0 and pc.layer_norm_grad_workspace(dtype, 1, 64) == 0
    lib = pc._load()
    assert lib.pconv_linear_workspace(pc.F16, 4, 5, 6, None) == pc.EINVAL
    n = ctypes.c_size_t(77)
    assert lib.pconv_linear_workspace(pc.F16, 4, 0, 6, ctypes.byref(n)) == pc.ESHAPE and n.value == 0


def test_the_convolutions_refuse_the_new_storage_type():
    pc.ensure_built()
    lib = pc._load()
    assert lib.pconv_maxpool2x2(X.at, Y.at, pc.BF16, 1, 1, 4, 4, None) == pc.EINVAL
    assert lib.pconv_dense_conv3x3(X.at, Y.at, W.at, None, pc.BF16, 1, 1, 1, 4, 4, 1, 1, 0, None) == pc.EINVAL
