"""The residual addition with RMS norm on the GPU against its float64 definition:
row and channel counts around the widths where kernels change, both residual
types, 8-bit outputs, gradients, refusals, streams and capture."""
import pytest
import torch

from oracle import mixer
from tests.mixer_harness import DTYPES, TOL, Draw, announce, check, ssd, streams_and_graphs
from tests.test_gpu_parity import _gpu  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 7), (1, 8), (2, 9), (5, 513), (3, 2048), (2, 2049), (1030, 511), (1030, 513), (1025, 1537),
          (1024, 2560), (1024, 4096), (1024, 4097), (3, 10241), (2, 16384), (2, 16385), (3, 24577), (2, 32768)]
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


def inputs(rows, C, dtype, residual, seed=3):
    n = Draw(seed)
    return {"x": n(rows, C, dtype=DTYPES[dtype]), "weight": 1 + n(C, scale=0.1),
            "residual": n(rows, C, scale=2.0, dtype=DTYPES[residual])}


@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("rows,C", SHAPES)
def test_forward_and_gradients(rows, C, dtype, residual):
    announce("add_norm %d x %d %s, residual %s" % (rows, C, dtype, residual))
    i = inputs(rows, C, dtype, residual)
    y, r = ssd.add_norm(**i)
    want_y, want_r = mixer.add_norm(i["x"], i["weight"], i["residual"], 1e-5)
    check("y", y, want_y)
    check("r", r, want_r)
    assert r.dtype == i["residual"].dtype and y.dtype == i["x"].dtype
    n = Draw(4)
    dy, dr = n(rows, C, dtype=y.dtype), n(rows, C, dtype=r.dtype)
    g = ssd.add_norm_backward(dy, r, i["weight"], dresidual=dr)
    want = mixer.add_norm_backward(dy, r, i["weight"], dr, 1e-5)
    for k in g:
        check(k, g[k], want[k])
    assert g["dx"].dtype == dy.dtype and g["dresidual"].dtype == r.dtype
    bare = ssd.add_norm_backward(dy, r)
    want = mixer.add_norm_backward(dy, r, None, None, 1e-5)
    assert bare["dweight"] is None
    # dx = rstd g - rstd n mean(g n): with one channel the second term is the first
    # times r^2 / (r^2 + eps), and what is left 1e-5 of either.  Each term is off by up
    # to 2,048 roundings of its own size, so dx by as much of the larger term, whatever
    # is left of it (the result's own rounding is of what is left).
    f = dy.cpu().double() / torch.sqrt(r.cpu().double().square().mean(-1, keepdim=True) + 1e-5)
    check("dx alone", bare["dx"], want["dx"],
          TOL[dy.dtype] + TOL[torch.float32] * float(f.abs().max() / want["dx"].abs().max()))


@pytest.mark.parametrize("to", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("dtype,residual", TYPES)
@pytest.mark.parametrize("rows,C", SHAPES)
def test_8_bits(rows, C, dtype, residual, to):
    announce("add_norm_q8 %d x %d %s, residual %s, %s" % (rows, C, dtype, residual, to))
    i = inputs(rows, C, dtype, residual)
    q, scale, r = ssd.add_norm_q8(**i, dtype=to)
    want, want_r = mixer.add_norm(i["x"], i["weight"], i["residual"], 1e-5)
    check("r", r, want_r)
    top = 127.0 if to is torch.int8 else 448.0
    m = want.abs().amax(-1)
    check("scale", scale, m / top)
    # half a step of the type: of 127 steps for the row's largest value (int8), of the
    # value itself or of the smallest normal's step (e4m3: 3 bits, 2^-6), and the
    # product's float32 roundings
    t = want / m[:, None] * top
    half = torch.full_like(t, 0.5) if to is torch.int8 else torch.clamp(t.abs() * 2.0 ** -4, min=2.0 ** -10)
    assert torch.all((q.float().cpu().double() - t).abs() <= half + top * 16 * 2.0 ** -24)
    # the quotient's rounding is exact: products and quotient in float32, one by one
    p = (i["x"].float() + i["residual"].float()) * i["weight"]
    quot = p / p.abs().amax(-1, keepdim=True) * top
    whole = torch.round(quot).to(torch.int8) if to is torch.int8 else quot.to(to)
    assert torch.equal(q.view(torch.uint8), whole.view(torch.uint8))


def test_without_residual_and_weight():
    announce("add_norm without residual, weight; more dimensions")
    x = Draw(1)(2, 3, 70).bfloat16()
    want, want_r = mixer.add_norm(x, None, None, 1e-5)
    y, r = ssd.add_norm(x)
    assert r is x and y.shape == x.shape
    check("y", y, want)
    y, r = ssd.add_norm(x, residual_dtype=torch.float32)
    assert torch.equal(r, x.float())
    q, scale, r = ssd.add_norm_q8(x)
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape and scale.shape == (2, 3) and r is x
    check("q scale", q.float() * scale[..., None], want, 2.0 ** -4 + TOL[torch.float32])


@pytest.mark.parametrize("to", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows", [5, 1100])
def test_rows_of_zeros_and_rows_that_are_not_finite(rows, to):
    announce("add_norm_q8: odd rows (%d)" % rows)
    i = inputs(rows, 300, "f32", "f32")
    i["x"][1] = 0
    i["residual"][1] = 0
    i["x"][2, 299] = float("nan")
    i["x"][3, 0] = float("inf")
    i["x"][4] = 1e20                     # its squares overflow
    q, scale, _ = ssd.add_norm_q8(**i, dtype=to)
    assert scale[1] == 0 and torch.all(q[1].float() == 0)
    assert torch.all(torch.isnan(scale[2:5])) and torch.all(q[2:5].float() == 0)
    keep = [k for k in range(rows) if k not in (2, 3, 4)]
    assert torch.all(torch.isfinite(scale[keep]))
    y, _ = ssd.add_norm(**i)
    assert torch.all(y[1] == 0) and torch.all(torch.isnan(y[2]))


def test_in_place_residual():
    """The C entry point with the residual updated in place."""
    import ctypes

    announce("add_norm in place")
    i = inputs(40, 520, "bf16", "f32")
    want_y, want_r = ssd.add_norm(**i)
    y = torch.empty_like(i["x"])
    prob = ssd.SsdNormProblem(40, 520, ssd.SSD_DTYPE_BF16, ssd.SSD_DTYPE_F32, ssd.SSD_DTYPE_BF16, 1e-5)
    rc = ssd.load_library().ssd_add_norm(
        ctypes.byref(prob), i["x"].data_ptr(), i["residual"].data_ptr(), i["weight"].data_ptr(), y.data_ptr(), None,
        i["residual"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == ssd.SSD_OK
    assert torch.equal(y, want_y) and torch.equal(i["residual"], want_r)


def test_refusals():
    announce("add_norm refusals")
    i = inputs(4, 24, "bf16", "f32")
    r = i["residual"]

    def refuse(error, call, **change):
        with pytest.raises(error):
            call(**{**i, **change})

    for call in (ssd.add_norm, ssd.add_norm_q8):
        refuse(TypeError, call, x=i["x"].half())
        refuse(ValueError, call, x=i["x"].cpu())
        refuse(ValueError, call, x=i["x"].t().contiguous().t())
        refuse(TypeError, call, weight=i["weight"].bfloat16())
        refuse(ValueError, call, weight=i["weight"][:8])
        refuse(TypeError, call, residual=r.double())
        refuse(ValueError, call, residual=r[:2])
        refuse(TypeError, call, residual_dtype=torch.bfloat16)
        refuse(ssd.SsdError, call, eps=-1.0)
        refuse(ssd.SsdError, call, eps=float("inf"))
    refuse(TypeError, ssd.add_norm, x=i["x"].float(), residual=r.bfloat16())
    refuse(TypeError, ssd.add_norm_q8, dtype=torch.uint8)
    with pytest.raises(ssd.SsdError) as e:
        ssd.add_norm(torch.zeros(2, 32769).cuda())
    assert e.value.code == ssd.SSD_ERR_UNSUPPORTED_DIMS
    with pytest.raises(ssd.SsdError) as e:
        ssd.add_norm(torch.zeros(0, 8).cuda())
    assert e.value.code == ssd.SSD_ERR_BAD_SHAPE
    with pytest.raises(TypeError):
        ssd.add_norm_backward(i["x"], r, i["weight"], dresidual=r.bfloat16())
    with pytest.raises(ValueError):
        ssd.add_norm_backward(i["x"], r, i["weight"], workspace=torch.empty(8, dtype=torch.uint8).cuda())


def test_streams_and_capture():
    announce("add_norm on a side stream and captured")
    for rows in (3, 1500):
        i = inputs(rows, 300, "bf16", "f32")
        dy = Draw(5)(rows, 300).bfloat16()
        streams_and_graphs(lambda: ssd.add_norm(**i))
        streams_and_graphs(lambda: ssd.add_norm_q8(**i, dtype=torch.int8))
        streams_and_graphs(lambda: ssd.add_norm_backward(dy, i["residual"], i["weight"]))


def test_more_rows_than_one_launch_dimension():
    rows = (1 << 32) // 64 + 1000     # (a launch's dimension has 32 bits of threads, 64 a row)
    announce("add_norm %d x 3" % rows)
    x = torch.zeros(rows, 3, dtype=torch.bfloat16).cuda()
    at = torch.cat([torch.arange(500), torch.arange((1 << 26) - 500, (1 << 26) + 500), torch.arange(rows - 500, rows)])
    x[at.cuda()] = Draw(6)(len(at), 3, dtype=torch.bfloat16)
    y, r = ssd.add_norm(x, torch.ones(3).cuda())
    want, _ = mixer.add_norm(x[at.cuda()], torch.ones(3).cuda(), None, 1e-5)
    check("y", y[at.cuda()], want)
    assert int((y != 0).any(-1).sum()) <= len(at)
    q, scale, _ = ssd.add_norm_q8(x, dtype=torch.int8)
    some, s, _ = ssd.add_norm_q8(x[at.cuda()], dtype=torch.int8)
    assert torch.equal(q[at.cuda()], some) and torch.equal(scale[at.cuda()], s)
