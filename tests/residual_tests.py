"""Tests of the sum behind a block (gate, residual, norms) that run on the GPU (test_queries_gpu.py) and on host threads
(test_queries_cpu.py): `bench` is the context under test.

Tolerances, derived before the first run, e = 2^-24, u the result type's rounding, D channels. A norm's sums are off by D / 4 e relative
(D terms dealt out to lanes; the mean's error enters the differences as D / 4 e of the mean absolute value), its root and products by 8 e: T =
(D / 4 + 16) e times what the largest number of the row would be. r adds products rounded to e each (and a hyperbolic tangent of 4 e). In h an
error t of r counts divided by the root, twice (by itself and in the root). Results are rounded once: u."""
import math

import pytest
import torch

from tests import cache_cases as C
from tests.cache_cases import E, INF, TYPES, U, close


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _norm(z, tol, norm, dtype):
    """(rows in 64 bits, tolerance) of a norm (kind, weight, bias, eps) or None of z, which is off by tol."""
    if norm is None:
        return z, tol
    kind, weight, bias, eps = norm
    D = z.shape[1]
    size = z.abs().amax(1, keepdim=True)
    if kind == "layer":
        z = z - z.mean(1, keepdim=True)
    root = (z.square().mean(1, keepdim=True) + eps).sqrt()
    w = 1.0 if weight is None else weight.double()
    tol = (2 * tol.amax(1, keepdim=True) + (D / 4 + 16) * E * 2 * size) / root * (1.0 if weight is None else w.abs()) * (1 + z.abs() / root)
    z = z / root * w
    return (z if bias is None else z + bias.double()), tol + 2 * E * (0.0 if bias is None else bias.double().abs()) + 2 * E * z.abs()


def _reference(x, y, gate, tanh, scale, post, pre, dtype):
    u = U[dtype] * (1 + 2 ** -6)
    least = 2.0 ** -25 if dtype == "f16" else 2.0 ** -133 if dtype == "bf16" else 2.0 ** -140
    r, tol = scale * x.double(), 2 * E * (scale * x.double()).abs()
    if y is not None:
        z, t = _norm(y.double(), torch.zeros(y.shape, dtype=torch.float64), post, dtype)
        g = torch.ones(1, 1, dtype=torch.float64) if gate is None else gate.double().tanh() if tanh else gate.double()
        r, tol = r + g * z, tol + g.abs() * t + 8 * E * (g * z).abs() + 2 * E * (r.abs() + (g * z).abs())
    h, h_tol = _norm(r, tol, pre, dtype)
    return (r, tol + u * r.abs() + least), (h, h_tol + u * h.abs() + least)


def _norms(kind, D, gen, dtype, with_weight=True):
    if kind == "none":
        return None
    t = TYPES[dtype]
    return (kind, (1 + 0.2 * torch.randn(D, generator=gen)).to(t) if with_weight else None,
            (0.2 * torch.randn(D, generator=gen)).to(t) if kind == "layer" and with_weight else None, 1e-5)


def _run(bench, x, y, gate, tanh, scale, post, pre, r, h):
    lib = bench.lib
    kinds = {"rms": lib.STTM_NORM_RMS, "layer": lib.STTM_NORM_LAYER}
    norm = lambda n: None if n is None else lib.Norm(kinds[n[0]], bench.put(n[1]), bench.put(n[2]), n[3])   # noqa: E731
    bench.ctx.sttm_residual_norm(x, y, r, h, post=norm(post), pre=norm(pre), gate=bench.put(gate), gate_tanh=tanh, scale=scale)
    bench.done()


RESIDUAL = [
    # dtype, n, width, post, pre, gate, tanh, scale
    ("bf16", 1, 3584, "rms", "rms", "one", True, 1.0),
    ("f32", 3, 1152, "layer", "layer", "row", False, 0.5),
    ("f16", 5, 8, "rms", "layer", "channel", True, 1.0),
    ("bf16", 9, 520, "none", "rms", "full", False, -1.5),
    ("f32", 2, 8192, "rms", "none", "none", False, 1.0),
    ("f16", 2, 16384, "layer", "rms", "channel", False, 1.0),
    ("f32", 1, 16384, "layer", "rms", "row", True, 1.0),
    ("bf16", 4, 4104, "rms", "rms", "full", True, 0.7071),
    ("bf16", 6, 1024, "none", "none", "one", False, 0.0),
    ("f32", 7, 24, "rms", "rms", "one", False, 1.0),
    ("f16", 3, 2048, "layer", "layer", "none", False, 1.0),
    ("bf16", 2, 1368, "layer", "rms", "row", True, 2.0),
]


@pytest.mark.parametrize("case", RESIDUAL, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("form", ["apart", "r_is_x_h_is_y", "r_is_y", "gaps"])
def test_residual_norm(bench, case, form):
    dtype, n, D, post, pre, gate, tanh, scale = case
    gen, t = _gen(D + n), TYPES[dtype]
    wide = D + 16 if form == "gaps" else D
    x, y = (torch.randn(n, wide, generator=gen).to(t) for _ in range(2))
    x = (x * 3 + 0.5).to(t)
    shape = {"none": None, "one": (1, 1), "row": (n, 1), "channel": (1, D), "full": (n, D)}[gate]
    g = None if shape is None else (0.8 * torch.randn(shape, generator=gen)).to(t)
    post, pre = _norms(post, D, gen, dtype), _norms(pre, D, gen, dtype, with_weight=form != "r_is_y")
    want = _reference(x[:, :D], y[:, :D], g, tanh, scale, post, pre, dtype)
    xd, yd = bench.guarded(x), bench.guarded(y)
    rd = xd if form == "r_is_x_h_is_y" else yd if form == "r_is_y" else bench.guarded(torch.full_like(x, 5.0))
    hd = yd if form == "r_is_x_h_is_y" else bench.guarded(torch.full_like(x, 5.0))
    _run(bench, xd[:, :D], yd[:, :D], g, tanh, scale, post, pre, rd[:, :D], hd[:, :D])
    close(rd[:, :D], *want[0], what="r")
    close(hd[:, :D], *want[1], what="h")
    if form == "gaps":
        assert (rd[:, D:] == 5).all() and (hd[:, D:] == 5).all() and torch.equal(xd.cpu(), x) and torch.equal(yd.cpu(), y)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 4160)])
def test_residual_norm_with_parts_left_out(bench, dtype, D):
    """No y (the first norm of a model), no h (the last sum), no r."""
    gen, n = _gen(D), 3
    x, y = (torch.randn(n, D, generator=gen).to(TYPES[dtype]) for _ in range(2))
    pre = _norms("rms", D, gen, dtype)
    want = _reference(x, None, None, False, 1.0, None, pre, dtype)
    h = bench.guarded(torch.zeros_like(x))
    _run(bench, bench.put(x), None, None, False, 1.0, None, pre, None, h)
    close(h, *want[1], what="h")
    r = bench.guarded(torch.zeros_like(x))
    want = _reference(x, y, None, False, 1.0, pre, None, dtype)
    _run(bench, bench.put(x), bench.put(y), None, False, 1.0, pre, None, r, None)
    close(r, *want[0], what="r")
    both = [bench.guarded(torch.zeros_like(x)) for _ in range(2)]
    _run(bench, bench.put(x), bench.put(y), None, False, 1.0, pre, None, *both)          # without a norm h is r
    assert torch.equal(both[0], r) and torch.equal(both[1], r)


def test_residual_norm_of_rows_that_are_not_finite(bench):
    """An infinity or NaN stays in its row; a row of zeros gives its bias; a constant row has no variance."""
    gen, D = _gen(3), 72
    x, y = torch.zeros(5, D), torch.randn(5, D, generator=gen)
    y[0, 5], y[1, 7], y[2], y[3] = INF, math.nan, 0.0, 3.0
    post = ("layer", torch.ones(D), torch.full((D,), 0.25), 1e-6)
    r, h = (bench.guarded(torch.zeros(5, D)) for _ in range(2))
    _run(bench, bench.put(x), bench.put(y), None, False, 1.0, post, ("rms", None, None, 1e-6), r, h)
    r, h = r.cpu(), h.cpu()
    assert torch.isnan(r[0]).any() and torch.isnan(r[1]).all() and torch.isnan(h[1]).all()
    assert (r[2] == 0.25).all() and (r[3] - 0.25).abs().max() < 1e-2 and torch.isfinite(r[2:]).all() and torch.isfinite(h[2:]).all()


def test_refusals_of_residual_norm(bench):
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731

    def refused(code, *args, **kw):
        with pytest.raises(lib.SttmError) as e:
            ctx.sttm_residual_norm(*args, **kw)
        assert e.value.code == code, e.value

    x, r, h = z(3, 64), z(3, 64), z(3, 64)
    refused(lib.STTM_ERR_SHAPE, z(3, 12), None, z(3, 12), None)
    refused(lib.STTM_ERR_SHAPE, z(3, 16392), None, z(3, 16392), None)
    refused(lib.STTM_ERR_SHAPE, z(64), None, r, h)
    refused(lib.STTM_ERR_SHAPE, x, z(2, 64), r, h)
    refused(lib.STTM_ERR_SHAPE, x, x, z(64, 3).T, h)
    refused(lib.STTM_ERR_SHAPE, z(3, 66)[:, :64], None, r, h)
    refused(lib.STTM_ERR_DTYPE, x, x.half(), r, h)
    refused(lib.STTM_ERR_DTYPE, x.long(), None, r, h)
    refused(lib.STTM_ERR_SHAPE, x, x, r, h, gate=z(2, 1))
    refused(lib.STTM_ERR_SHAPE, x, x, r, h, gate=z(64))
    refused(lib.STTM_ERR_DTYPE, x, x, r, h, gate=z(1, 1).half())
    refused(lib.STTM_ERR_SHAPE, x, x, r, h, gate=z(3, 66)[:, :64])
    refused(lib.STTM_ERR_ARG, x, None, r, h, gate=z(1, 1))
    refused(lib.STTM_ERR_ARG, x, None, r, h, post=lib.Norm(lib.STTM_NORM_RMS))
    refused(lib.STTM_ERR_ARG, x, x, r, None, pre=lib.Norm(lib.STTM_NORM_RMS))
    refused(lib.STTM_ERR_ARG, x, x, r, r)
    refused(lib.STTM_ERR_NULL, x, x, None, None)
    refused(lib.STTM_ERR_ARG, x, x, r, h, scale=math.nan)
    refused(lib.STTM_ERR_ARG, x, x, r, h, pre=lib.Norm(2))
    refused(lib.STTM_ERR_ARG, x, x, r, h, pre=lib.Norm(lib.STTM_NORM_RMS, eps=-1.0))
    refused(lib.STTM_ERR_SHAPE, x, x, r, h, pre=lib.Norm(lib.STTM_NORM_RMS, z(32)))
    refused(lib.STTM_ERR_DTYPE, x, x, r, h, pre=lib.Norm(lib.STTM_NORM_RMS, z(64).half()))
    refused(lib.STTM_ERR_ARG, x, x, r, h, pre=lib.Norm(lib.STTM_NORM_RMS, z(65)[1:]))
    refused(lib.STTM_ERR_ARG, z(3 * 64 + 1)[1:].view(3, 64), None, r, h)
    with pytest.raises(lib.SttmError):
        lib.Norm(lib.STTM_NORM_RMS, z(2, 32))
    ctx.sttm_residual_norm(z(0, 64), z(0, 64), z(0, 64), None)              # no rows: nothing to do
    bench.done()
