"""The operators around the layer on the GPU, every value by its own size: a value may be
off by as many roundings as ``TOL`` allows of the sum of its terms' magnitudes (and by
its own type's rounding), however large others of its tensor are.

The same 2,048 roundings hold here: a decay exp(-c) that still counts has c <= 87, off by
4 roundings of A, 4 of the time step and 2 of their product, 10 x 87 in all; a term passes
through at most T <= 900 sums (and as many products with decays near 1, each off by its
rounding only where c is small); sums over channels, rows and chunks add fewer than 200."""
import pytest
import torch

from oracle import mixer
from tests.mixer_harness import DTYPES, TOL, Draw, announce, seq_idx_of, ssd
from tests.test_gpu_add_norm import inputs as norm_inputs
from tests.test_gpu_conv import inputs as conv_inputs
from tests.test_gpu_parity import _gpu  # noqa: F401
from tests.test_gpu_scan import inputs as scan_inputs

pytestmark = pytest.mark.gpu


def each(name, got, want, size):
    """|got - want| against the value's own sum of magnitudes and its type's rounding."""
    assert got.shape == want.shape == size.shape, name
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    # (decays, and SiLU's exponentials, below 2^-126 may count as 0)
    allowed = TOL[torch.float32] * size.double() + half * want.abs() + 2.0 ** -110
    bad = ~((got.detach().double().cpu() - want).abs() <= allowed)
    assert not bad.any(), "%s: %d of %d" % (name, bad.sum(), bad.numel())


def plus(t):
    return None if t is None else t.detach().double().cpu().abs()


def slope_size(v):
    """The magnitudes that SiLU's derivative s (1 + v (1 - s)) is made of."""
    s = torch.sigmoid(v)
    return s * (1 + v.abs() * (1 - s))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,T,E,N,G,starts", [
    (1, 1, 64, 16, 1, None), (2, 130, 70, 16, 1, None), (1, 900, 80, 32, 2, None), (4, 300, 200, 16, 1, None),
    (1, 300, 64, 128, 1, None), (1, 900, 130, 32, 2, [0, 2, 300, 301, 304, 880, 900]), (1, 700, 66, 16, 1, [0, 1, 500, 501, 700])])
def test_scan(b, T, E, N, G, starts, dtype):
    announce("scan, value by value: b%d T%d E%d N%d G%d %s starts %s" % (b, T, E, N, G, dtype, starts))
    spans = mixer.packed(starts) if starts else mixer.rows(b, T)
    i = scan_inputs(b, T, E, N, G, dtype, len(spans))
    seq = {"seq_idx": seq_idx_of(starts), "nseq": len(spans)} if starts else {}
    n = Draw(4)
    dy, df = n(b, T, E, dtype=DTYPES[dtype]), n(len(spans), E, N)
    names = {"softplus": True, "init": i["initial_states"], "spans": spans,
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C", "D", "z", "dt_bias")}}
    want_y, want_f = mixer.scan_forward(**names)
    want = mixer.scan_backward(**names, dy=dy, dfinal=df)

    # the same sums of magnitudes: without the gate, which is a factor of y and dy
    z = i["z"].double().cpu()
    gate = z * torch.sigmoid(z)
    sizes = {**names, **{k: plus(names[k]) for k in ("x", "B", "C", "D", "init")}, "z": None}
    size_y, size_f = mixer.scan_forward(**sizes)
    dyg = plus(dy) * gate.abs()
    size = mixer.scan_backward(**sizes, dy=dyg, dfinal=plus(df))
    _, v, d, _, _, _, D, _ = mixer._scan_inputs(*(sizes[k] for k in ("x", "dt", "A_log", "B", "C", "D", "dt_bias")), True)
    xdu, s = (size["dx"] - D * dyg) / d * sizes["x"], torch.sigmoid(v)
    size["ddt"] = (2 * xdu - size["ddt"] / s) * s    # (the product with A is negative)
    size["ddt_bias"] = size["ddt"].sum((0, 1))
    size["dA_log"] = -size["dA_log"]
    size["dz"] = plus(dy) * size_y * slope_size(z)

    y, f = ssd.scan_forward(**i, **seq)
    each("y", y, want_y, size_y * gate.abs())
    each("final", f, want_f, size_f)
    g = ssd.scan_backward(**i, dy=dy, dfinal_states=df, **seq)
    for k in g:
        each(k, g[k], want[k], size[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,T,C,W,starts", [(2, 50, 70, 4, None), (1, 300, 33, 2, None),
                                            (1, 300, 130, 4, [0, 1, 2, 100, 103, 290, 300])])
def test_conv(b, T, C, W, starts, dtype):
    announce("conv, value by value: b%d T%d C%d W%d %s starts %s" % (b, T, C, W, dtype, starts))
    spans = mixer.packed(starts) if starts else mixer.rows(b, T)
    i = conv_inputs(b, T, C, W, dtype, len(spans), True, False)
    seq = {"seq_idx": seq_idx_of(starts), "nseq": len(spans)} if starts else {}
    x, w, bias, init = i["x"], i["weight"], i["bias"], i["initial_states"]
    n = Draw(4)
    dy, df = n(b, T, C, dtype=x.dtype), n(len(spans), W - 1, C, dtype=x.dtype)
    want_y, want_f = mixer.conv_forward(x, w, bias, True, init, spans)
    want = mixer.conv_backward(x, w, bias, True, init, spans, dy, df)
    # SiLU is no steeper than 1.1, its derivative than 0.5
    v, _ = mixer.conv_forward(x, w, bias, False, init, spans)
    size_v, _ = mixer.conv_forward(plus(x), plus(w), plus(bias), False, plus(init), spans)
    size = mixer.conv_backward(plus(x), plus(w), plus(bias), False, plus(init), spans, plus(dy) * (slope_size(v) + size_v), plus(df))
    y, f = ssd.conv_forward(**i, **seq)
    each("y", y, want_y, 1.1 * size_v)
    assert torch.equal(f.double().cpu(), want_f)
    g = ssd.conv_backward(x, w, dy, bias=bias, initial_states=init, dfinal_states=df, **seq)
    for k in g:
        each(k, g[k], want[k], size[k])


@pytest.mark.parametrize("dtype,residual", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,C", [(3, 7), (37, 513), (65, 2560), (3, 10241), (3, 24577)])
def test_norm(rows, C, dtype, residual):
    announce("add_norm, value by value: %d x %d %s, residual %s" % (rows, C, dtype, residual))
    i = norm_inputs(rows, C, dtype, residual)
    i["x"][0] *= 1e-3        # (rows of other sizes than the largest)
    i["residual"][0] *= 1e-3
    y, r = ssd.add_norm(**i)
    want_y, want_r = mixer.add_norm(i["x"], i["weight"], i["residual"], 1e-5)
    each("y", y, want_y, want_y.abs())
    each("r", r, want_r, want_r.abs())
    n = Draw(4)
    dy, dr = n(rows, C, dtype=y.dtype), n(rows, C, dtype=r.dtype)
    g, want = ssd.add_norm_backward(dy, r, i["weight"], dresidual=dr), mixer.add_norm_backward(dy, r, i["weight"], dr, 1e-5)
    rr, gw = plus(r), plus(dy) * plus(i["weight"])
    rstd = 1 / torch.sqrt(rr.square().mean(-1, keepdim=True) + 1e-5)
    size = rstd * (gw + rr * rstd * (gw * rr * rstd).mean(-1, keepdim=True)) + plus(dr)
    each("dx", g["dx"], want["dx"], size)
    each("dresidual", g["dresidual"], want["dresidual"], size)
    each("dweight", g["dweight"], want["dweight"], (plus(dy) * rr * rstd).sum(0))
