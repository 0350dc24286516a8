"""Layer norm and its gradient: against the formulas in 64 bits, against differences, and what the calls refuse."""
import ctypes
import math

import pytest
import torch

from paper_2605_26636_b200 import build as jv_build
from paper_2605_26636_b200 import jetvit as jv
from tests._util import guarded_empty

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # a rounding is off by at most half a step
U = 2.0 ** -24


def _inputs(rows, C, dtype, seed=0, offset=0.3, device="cuda"):
    g = torch.Generator().manual_seed(1000 * seed + rows + C)
    x = (torch.randn(rows, C, generator=g) * torch.exp(0.5 * torch.randn(C, generator=g)) + offset).to(dtype).to(device)
    dy = torch.randn(rows, C, generator=g).to(dtype).to(device)
    w, b = (1 + 0.3 * torch.randn(C, generator=g)).to(device), (0.2 * torch.randn(C, generator=g)).to(device)
    return x, dy, w, b


def _reference(x, w, b, eps):
    """y in 64 bits, and what the arithmetic of the kernel may add to a rounding of it: sums of up to 32 values a lane, a tree
    of 32 lanes and up to 16 warps (64 roundings at most) in the mean and the variance."""
    x, w, b = x.double(), w.double(), b.double()
    mean = x.mean(-1, keepdim=True)
    rstd = (((x - mean) ** 2).mean(-1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * rstd
    bound = 64 * U * (w.abs() * (xh.abs() + rstd * x.abs().mean(-1, keepdim=True)) + b.abs())
    return xh * w + b, bound, mean[..., 0], rstd[..., 0]


# columns: one, odd, each count of 16-byte pieces a lane with a remainder, the longest row of a warp, rows of a block
COLS = [1, 7, 8, 33, 264, 384, 520, 776, 1023, 1024, 1032, 2048, 5000, 16384]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", COLS)
def test_forward(C, dtype):
    for rows in (1, 5, 263):
        x, _, w, b = _inputs(rows, C, dtype)
        out, check = guarded_empty((rows, C), dtype, "cuda")
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        y = jv.layer_norm(x, w, b, eps=1e-5, out=out, stats=(mean, rstd))
        check()
        ref, bound, m, r = _reference(x, w, b, 1e-5)
        assert ((y.double() - ref).abs() <= HALF[dtype] * (ref.abs() + bound) + bound).all()
        assert ((mean.double() - m).abs() <= 64 * U * x.double().abs().mean(-1)).all()
        assert ((rstd.double() - r).abs() <= 64 * U * r * (1 + (r * x.double().abs().mean(-1)) ** 2 * U)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", [7, 384, 1024, 1032, 5000])
@pytest.mark.parametrize("size,eps", [(1e20, 1e-5), (1e30, 0.0), (1e37, 1e-5), (1e-18, 0.0), (1e-25, 1e-38)])
def test_variances_that_leave_fp32(C, dtype, size, eps):
    """Every other row far larger, or smaller, than its squares in fp32 allow, two rows of bf16 to a warp among them; a row of one value
    beside them."""
    for rows in (5, 5001):
        x, _, w, b = _inputs(rows, C, dtype, seed=4, offset=0.0)
        x[::2] = (x[::2].float() * size).to(dtype)
        if eps > 0.0:
            x[1] = 3.0
        stats = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        y = jv.layer_norm(x, w, b, eps=eps, stats=stats)
        ref, bound, m, r = _reference(x, w, b, eps)
        assert ((y.double() - ref).abs() <= HALF[dtype] * (ref.abs() + bound) + bound).all()
        assert ((stats[0].double() - m).abs() <= 64 * U * x.double().abs().mean(-1)).all()
        # (1 / standard deviation itself is a small, or large, fp32 number: within 2^-126 it has fewer bits)
        assert ((stats[1].double() - r).abs() <= (64 * U * r * (1 + (r * x.double().abs().mean(-1)) ** 2 * U) + 2.0 ** -149)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", COLS)
def test_gradient(C, dtype):
    for rows in (1, 6, 2500 if C <= 2048 else 700):
        x, dy, w, _ = _inputs(rows, C, dtype, seed=1)
        _, _, m, r = _reference(x, w, w, 1e-5)
        mean, rstd = m.float(), r.float()
        dx, dw, db = jv.layer_norm_grad(dy, x, w, mean, rstd)
        xd, d, m, r = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
        xh, g = (xd - m) * r, d * w.double()
        mg, mgx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        ref = r * (g - mg - xh * mgx)
        # the two means: 70 roundings at most; what follows them and forms xh: six; (x - mean) is formed from the given fp32 mean
        bound = U * r * (6 * (g.abs() + mg.abs() + (xh * mgx).abs()) +
                         70 * (g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)))
        assert ((dx.double() - ref).abs() <= HALF[dtype] * (ref.abs() + bound) + bound).all()
        # a column's sum: rows of a warp one after the other (at least 148 blocks), its block's warps, the blocks' partials
        depth = rows / 148 + 1 + 4 + 3 * 148 / 8 + 1 + 8 + 4
        assert ((dw.double() - (d * xh).sum(0)).abs() <= depth * U * (d * xh).abs().sum(0) + 1e-30).all()
        assert ((db.double() - d.sum(0)).abs() <= depth * U * d.abs().sum(0) + 1e-30).all()
        again = jv.layer_norm_grad(dy, x, w, mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))      # sums in a fixed order


@pytest.mark.gpu
def test_gradient_against_differences():
    """Of sum(dy * layer_norm(x)) in x, w and b: central differences of the forward pass itself, in fp32."""
    x, dy, w, b = _inputs(3, 40, torch.float32, seed=2)
    stats = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    jv.layer_norm(x, w, b, stats=stats)
    dx, dw, db = jv.layer_norm_grad(dy, x, w, *stats)
    f = lambda x, w, b: float((dy.double() * jv.layer_norm(x, w, b).double()).sum())
    h = 2.0 ** -6
    # outputs are off by some 64 U each, so a difference of two sums of 120 of them by less than 120 * 128 U * 4 / (2 h); the
    # third derivative of a normalised row adds h^2 times a small number
    tol = 120 * 128 * U * 4 / (2 * h) + 8 * h * h
    for grad, which in ((dx, 0), (dw, 1), (db, 2)):
        for i in range(0, grad.numel(), 7):
            args = [x.clone(), w.clone(), b.clone()]
            args[which].view(-1)[i] += h
            up = f(*args)
            args[which].view(-1)[i] -= 2 * h
            assert abs((up - f(*args)) / (2 * h) - float(grad.view(-1)[i])) <= tol


@pytest.mark.gpu
def test_strides_alignment_and_missing_vectors():
    x, dy, w, b = _inputs(37, 3 * 192, torch.bfloat16, seed=3)
    for lo, C in ((192, 192), (8, 64), (1, 191), (5, 64)):          # slices of wider rows: on and off 16-byte boundaries
        xs, ds = x[:, lo:lo + C], dy[:, lo:lo + C]
        stats = torch.empty(37, device="cuda"), torch.empty(37, device="cuda")
        y = jv.layer_norm(xs, w[:C].clone(), None, stats=stats)
        y0 = jv.layer_norm(xs.contiguous(), w[:C].clone(), torch.zeros(C, device="cuda"))
        ref, bound, _, _ = _reference(xs, w[:C], torch.zeros(C, device="cuda"), 1e-6)
        for t in (y, y0):
            assert ((t.double() - ref).abs() <= HALF[x.dtype] * (ref.abs() + bound) + bound).all()
        one = torch.ones(C, device="cuda")
        full = jv.layer_norm_grad(ds.contiguous(), xs.contiguous(), one, *stats)
        strided = jv.layer_norm_grad(ds, xs, None, *stats)
        step = 2 * HALF[x.dtype]
        assert ((full[0].double() - strided[0].double()).abs() <= step * full[0].double().abs() + 1e-5).all()
        for p, q in zip(full[1:], strided[1:]):
            assert ((p - q).abs() <= 1e-5 * p.abs() + 1e-4).all()
        dx, dw, db = jv.layer_norm_grad(ds, xs, None, *stats, weight_grad=False, bias_grad=False)
        assert dw is None and db is None and torch.equal(dx, strided[0])
        _, dw, none = jv.layer_norm_grad(ds, xs, None, *stats, bias_grad=False)
        assert none is None and torch.equal(dw, strided[1])
    big = torch.zeros(4, 5, 64, device="cuda", dtype=torch.bfloat16)
    assert jv.layer_norm(big).shape == big.shape
    wc = w[1:65]                                                        # weights off a 16-byte boundary
    y = jv.layer_norm(x[:, :64], wc)
    ref, bound, _, _ = _reference(x[:, :64], wc, torch.zeros(64, device="cuda"), 1e-6)
    assert ((y.double() - ref).abs() <= HALF[x.dtype] * (ref.abs() + bound) + bound).all()


@pytest.mark.gpu
def test_large_mean_constant_rows_and_values_that_are_none():
    C = 512
    x = torch.randn(4, C, device="cuda") * 0.01 + 300.0                # spread 1 / 30000 of the mean
    y = jv.layer_norm(x, eps=0.0)
    ref, bound, _, _ = _reference(x, torch.ones(C, device="cuda"), torch.zeros(C, device="cuda"), 0.0)
    assert ((y.double() - ref).abs() <= bound).all()
    const = torch.full((2, C), 7.25, device="cuda")
    assert (jv.layer_norm(const, eps=1e-6) == 0).all()
    bad = torch.randn(3, C, device="cuda")
    bad[1, 5] = math.nan
    bad[2, 6] = math.inf
    y = jv.layer_norm(bad)
    assert torch.isfinite(y[0]).all() and torch.isnan(y[1]).all() and torch.isnan(y[2]).all()


@pytest.mark.gpu
def test_rows_whose_offsets_pass_32_bits():
    C, rows, far = 264, 40, 1 << 26                             # elements between rows: 2^31 behind the 32nd
    x, dy, w, b = _inputs(rows, C, torch.bfloat16, seed=6)
    pool = torch.empty(far * (rows - 1) + 2 * C, dtype=torch.bfloat16, device="cuda")
    xs, ds = pool.as_strided((rows, C), (far, 1)), pool.as_strided((rows, C), (far, 1), C)
    xs.copy_(x)
    ds.copy_(dy)
    stats = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    assert torch.equal(jv.layer_norm(xs, w, b, stats=stats), jv.layer_norm(x, w, b))
    assert all(torch.equal(p, q) for p, q in zip(jv.layer_norm_grad(ds, xs, w, *stats), jv.layer_norm_grad(dy, x, w, *stats)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_rows(dtype):
    """Enough rows for two to a warp, their count odd, and for several to a warp of the gradient."""
    for rows, C in ((5001, 384), (9999, 1024), (7001, 129)):
        x, dy, w, b = _inputs(rows, C, dtype, seed=7)
        stats = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        out, check = guarded_empty((rows, C), dtype, "cuda")
        y = jv.layer_norm(x, w, b, eps=1e-5, out=out, stats=stats)
        check()
        ref, bound, m, r = _reference(x, w, b, 1e-5)
        assert ((y.double() - ref).abs() <= HALF[dtype] * (ref.abs() + bound) + bound).all()
        assert ((stats[0].double() - m).abs() <= 64 * U * x.double().abs().mean(-1)).all()
        one = [torch.cat([jv.layer_norm(x[i:i + 1], w, b, eps=1e-5) for i in (0, 1, rows - 1)])]
        assert torch.equal(one[0], y[[0, 1, rows - 1]])               # however many rows a call has


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    x, dy, w, b = _inputs(129, 384, torch.bfloat16, seed=4)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    stats = torch.empty(129, device="cuda"), torch.empty(129, device="cuda")
    dw, db = torch.empty(384, device="cuda"), torch.empty(384, device="cuda")
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    want = jv.layer_norm(x, w, b, stats=stats).clone()
    want_g = [t.clone() for t in jv.layer_norm_grad(dy, x, w, *stats)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = jv.layer_norm(x, w, b, stream=side)
    got_g = jv.layer_norm_grad(dy, x, w, *stats, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, c) for a, c in zip(got_g, want_g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jv.layer_norm(x, w, b, out=y, stats=stats)
        jv.layer_norm_grad(dy, x, w, *stats, out=(dx, dw, db), ws=ws)
    x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want.flip(0))
    assert torch.equal(dx, jv.layer_norm_grad(dy, x, w, *stats)[0])


# ---- refusals, on the host ------------------------------------------------------------------------------------------
X, W, Y, M, R, DY, WS = (i << 24 for i in range(1, 8))


@pytest.mark.gpu
def test_results_on_another_stream_do_not_lie_where_earlier_work_still_writes():
    """Memory that this stream has freed may have work ahead of it here; a call for another stream takes none of it."""
    x, dy, w, b = _inputs(4096, 512, torch.float32)
    stats = torch.empty(4096, device="cuda"), torch.empty(4096, device="cuda")
    want = jv.layer_norm(x, w, b, stats=stats)
    want_g = jv.layer_norm_grad(dy, x, w, *stats)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    late = [torch.empty_like(x) for _ in range(2)] + [torch.empty(512, device="cuda") for _ in range(2)]
    late.append(torch.empty(int(jv.lib().jv_layer_norm_grad_workspace_bytes(ctypes.byref(jv.JvNormShape(4096, 512, jv.JV_F32, 0, 0)))), dtype=torch.uint8, device="cuda"))
    torch.cuda._sleep(1 << 26)
    for t in late:
        t.fill_(7)
    del late, t
    got, got_g = jv.layer_norm(x, w, b, stream=side), jv.layer_norm_grad(dy, x, w, *stats, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, e) for a, e in zip(got_g, want_g))


@pytest.fixture(scope="module")
def L():
    jv_build.build()
    return jv.lib()


def _fwd(L, shp=jv.JvNormShape(8, 64, jv.JV_F32, 0, 0), x=X, w=W, b=None, y=Y, mean=M, rstd=R, eps=1e-6):
    return L.jv_layer_norm(x, w, b, y, mean, rstd, ctypes.byref(shp) if shp else None, eps, None)


def test_refusals(L):
    bad = jv.JV_ERR_INVALID_ARG
    S = jv.JvNormShape
    for kw in (dict(shp=None), dict(shp=S(0, 64, 0, 0, 0)), dict(shp=S(8, 0, 0, 0, 0)), dict(shp=S(8, 64, 2, 0, 0)), dict(shp=S(8, 64, 0, 63, 0)),
               dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(eps=-1.0), dict(eps=math.nan), dict(x=X + 2), dict(w=W + 2),
               dict(y=X), dict(y=X + 8 * 64 * 4 - 4), dict(y=W), dict(mean=Y + 4), dict(rstd=M)):
        assert _fwd(L, **kw) == bad, kw
    assert _fwd(L, shp=S(8, 16385, 0, 0, 0)) == jv.JV_ERR_UNSUPPORTED
    assert _fwd(L, shp=S(1 << 31, 64, 0, 0, 0)) == jv.JV_ERR_UNSUPPORTED
    for strides in ((1 << 31, 0), (0, 1 << 31)):                     # extents that 64 bits of bytes do not hold
        assert _fwd(L, shp=S((1 << 31) - 1, 64, 0, *strides)) == jv.JV_ERR_UNSUPPORTED
    shp = S(8, 64, jv.JV_F32, 0, 0)
    need = L.jv_layer_norm_grad_workspace_bytes(ctypes.byref(shp))
    assert need >= 2 * 64 * 4 and L.jv_layer_norm_grad_workspace_bytes(ctypes.byref(S(0, 64, 0, 0, 0))) == 0
    grad = lambda dy=DY, x=X, mean=M, rstd=R, dx=Y, dw=W + 4096, db=None, ws=WS, n=need, shp=shp: L.jv_layer_norm_grad(
        dy, x, W, mean, rstd, dx, dw, db, ctypes.byref(shp), ws, n, None)
    for kw in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(dx=DY), dict(dw=Y), dict(db=W + 4096),
               dict(ws=Y), dict(shp=S(8, 64, 0, 0, 1))):
        assert grad(**kw) == bad, kw
    for kw in (dict(ws=None), dict(ws=WS + 4), dict(n=need - 1)):
        assert grad(**kw) == jv.JV_ERR_WORKSPACE, kw
    if not torch.cuda.is_available():
        assert _fwd(L) in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)
        assert grad(dw=None, ws=None, n=0) in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)      # no sums wanted: no scratch


def test_binding_refuses_cpu_tensors_and_rows_that_are_not_rows():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        jv.layer_norm(x)
    with pytest.raises(ValueError):
        jv.layer_norm_grad(x, x, None, torch.zeros(4), torch.zeros(4))
