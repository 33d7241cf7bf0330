"""Host-side checks of the convolution's, the scan's and the norm's entry points:
invalid arguments are refused, with their codes, before anything touches the
device."""
import ctypes

import pytest
import torch

from paper_2405_21060_amd import ssd

FAKE = 0x10000   # never dereferenced: every call below fails validation first
ODD = FAKE + 2
BF16, F32 = ssd.SSD_DTYPE_BF16, ssd.SSD_DTYPE_F32


@pytest.fixture(scope="module")
def lib():
    return ssd.load_library()


def conv(parts=(5120, 128, 128), **kw):
    base = dict(batch=4, seqlen=4096, channels=5376, width=4, nseq=0, x_batch_stride=4096 * 5376, x_token_stride=5376,
                nparts=len(parts), dtype=BF16, silu=1)
    base.update(kw)
    return ssd.SsdConvProblem(parts=(ctypes.c_int64 * 3)(*(tuple(parts[:3]) + (0,) * (3 - len(parts[:3])))), **base)


def scan(**kw):
    base = dict(batch=4, seqlen=4096, channels=5120, dstate=16, ngroups=1, nseq=0, dtype=BF16, dt_softplus=1)
    base.update(kw)
    E, T, GN = base["channels"], base["seqlen"], base["ngroups"] * base["dstate"]
    for name, row in (("x", E), ("dt", E), ("z", E), ("b", GN), ("c", GN)):
        base.setdefault(name + "_batch_stride", T * row)
        base.setdefault(name + "_token_stride", row)
    return ssd.SsdScanProblem(**base)


def norm(**kw):
    base = dict(rows=16384, channels=2560, dtype=BF16, residual_dtype=F32, out_dtype=BF16, eps=1e-5)
    base.update(kw)
    return ssd.SsdNormProblem(**base)


def pointers(*at):
    return (ctypes.c_void_p * 3)(*at)


def conv_calls(lib, p, seq=None, x=FAKE, weight=FAKE, y=(FAKE, FAKE, FAKE), ws=FAKE, ws_bytes=1 << 40):
    p = ctypes.byref(p) if p is not None else None
    return (lib.ssd_conv_forward(p, x, weight, None, None, seq, pointers(*y), None, None),
            lib.ssd_conv_backward(p, x, weight, None, None, seq, pointers(*y), None, FAKE, FAKE, None, None, ws, ws_bytes, None))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), ssd.SSD_ERR_BAD_DTYPE), (dict(seqlen=0), ssd.SSD_ERR_BAD_SHAPE),
    (dict(batch=0), ssd.SSD_ERR_BAD_SHAPE), (dict(channels=0), ssd.SSD_ERR_BAD_SHAPE),
    (dict(width=1), ssd.SSD_ERR_UNSUPPORTED_DIMS), (dict(width=5), ssd.SSD_ERR_UNSUPPORTED_DIMS),
    (dict(x_token_stride=-1), ssd.SSD_ERR_BAD_SHAPE), (dict(x_batch_stride=-1), ssd.SSD_ERR_BAD_SHAPE),
    (dict(nparts=0), ssd.SSD_ERR_BAD_SHAPE), (dict(nparts=4), ssd.SSD_ERR_BAD_SHAPE),
    (dict(nparts=2), ssd.SSD_ERR_BAD_SHAPE),                          # the parts do not add up
    (dict(parts=(5120, 256, 0)), ssd.SSD_ERR_BAD_SHAPE), (dict(parts=(5120, 128, 129)), ssd.SSD_ERR_BAD_SHAPE),
    (dict(parts=(1 << 62, 1 << 62, 5376)), ssd.SSD_ERR_BAD_SHAPE),
    (dict(seqlen=1 << 40), ssd.SSD_ERR_TOO_LARGE), (dict(x_token_stride=1 << 50), ssd.SSD_ERR_TOO_LARGE)])
def test_conv_shapes(lib, kw, code):
    assert conv_calls(lib, conv(**kw)) == (code, code)
    size = ctypes.c_size_t(0)
    assert lib.ssd_conv_backward_workspace_bytes(ctypes.byref(conv(**kw)), ctypes.byref(size)) == code


def test_conv_arguments(lib):
    null, shape = ssd.SSD_ERR_NULL_ARG, ssd.SSD_ERR_BAD_SHAPE
    assert conv_calls(lib, None) == (null, null)
    assert conv_calls(lib, conv(), x=None) == (null, null)
    assert conv_calls(lib, conv(), weight=None) == (null, null)
    assert conv_calls(lib, conv(), y=(FAKE, None, FAKE)) == (null, null)
    batch = ssd.SSD_ERR_SEQIDX_BATCH
    assert conv_calls(lib, conv(nseq=3), seq=FAKE) == (batch, batch)
    for nseq in (0, -1, 4097):
        assert conv_calls(lib, conv(batch=1, nseq=nseq), seq=FAKE) == (shape, shape)
    size = ctypes.c_size_t(0)
    assert lib.ssd_conv_backward_workspace_bytes(ctypes.byref(conv()), ctypes.byref(size)) == ssd.SSD_OK
    assert lib.ssd_conv_backward_workspace_bytes(ctypes.byref(conv()), None) == null
    assert size.value >= 4 * 5376 * 5    # a row of partial sums at least
    assert conv_calls(lib, conv(), ws_bytes=size.value - 1)[1] == ssd.SSD_ERR_WORKSPACE
    assert conv_calls(lib, conv(), ws=None)[1] == ssd.SSD_ERR_WORKSPACE
    assert conv_calls(lib, conv(), ws=FAKE + 4)[1] == ssd.SSD_ERR_UNSUPPORTED_DIMS
    # a step has no tokens or parts to be wrong about
    step = lambda p, state=FAKE, x=FAKE: lib.ssd_conv_step(ctypes.byref(p), x, FAKE, None, state, FAKE, None)
    assert step(conv(seqlen=0, nparts=0, x_token_stride=-1), state=None) == null
    assert step(conv(), x=None) == null
    assert step(conv(width=5)) == ssd.SSD_ERR_UNSUPPORTED_DIMS
    assert step(conv(dtype=2)) == ssd.SSD_ERR_BAD_DTYPE


def scan_calls(lib, p, seq=None, x=FAKE, B=FAKE, z=None, init=None, A=FAKE, ws=FAKE, ws_bytes=1 << 40, dz=FAKE, dy=FAKE):
    p = ctypes.byref(p) if p is not None else None
    return (lib.ssd_scan_forward(p, x, FAKE, A, B, FAKE, None, z, None, init, seq, FAKE, None, ws, ws_bytes, None)
            if dy and dz else None,
            lib.ssd_scan_backward(p, x, FAKE, A, B, FAKE, None, z, None, init, seq, dy, None, FAKE, FAKE, FAKE, FAKE,
                                  FAKE, None, dz, None, None, ws, ws_bytes, None))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), ssd.SSD_ERR_BAD_DTYPE), (dict(seqlen=0), ssd.SSD_ERR_BAD_SHAPE),
    (dict(channels=5120, ngroups=3), ssd.SSD_ERR_BAD_SHAPE), (dict(ngroups=0), ssd.SSD_ERR_BAD_SHAPE),
    (dict(dstate=24), ssd.SSD_ERR_UNSUPPORTED_DIMS), (dict(dstate=272), ssd.SSD_ERR_UNSUPPORTED_DIMS),
    (dict(x_token_stride=-1), ssd.SSD_ERR_BAD_SHAPE), (dict(c_batch_stride=-2), ssd.SSD_ERR_BAD_SHAPE),
    (dict(seqlen=1 << 40), ssd.SSD_ERR_TOO_LARGE), (dict(b_token_stride=1 << 50), ssd.SSD_ERR_TOO_LARGE)])
def test_scan_shapes(lib, kw, code):
    assert scan_calls(lib, scan(**kw)) == (code, code)
    size = ctypes.c_size_t(0)
    assert lib.ssd_scan_workspace_bytes(ctypes.byref(scan(**kw)), ctypes.byref(size)) == code
    assert lib.ssd_scan_backward_workspace_bytes(ctypes.byref(scan(**kw)), ctypes.byref(size)) == code


def test_scan_arguments(lib):
    null, dims = ssd.SSD_ERR_NULL_ARG, ssd.SSD_ERR_UNSUPPORTED_DIMS
    assert scan_calls(lib, None) == (null, null)
    assert scan_calls(lib, scan(), x=None) == (null, null)
    assert scan_calls(lib, scan(), dy=None)[1] == null
    assert scan_calls(lib, scan(), z=FAKE, dz=None)[1] == null
    assert scan_calls(lib, scan(), B=ODD) == (dims, dims)
    assert scan_calls(lib, scan(b_token_stride=17)) == (dims, dims)
    assert scan_calls(lib, scan(c_batch_stride=17)) == (dims, dims)
    assert scan_calls(lib, scan(), A=FAKE + 4) == (dims, dims)
    assert scan_calls(lib, scan(), init=FAKE + 8) == (dims, dims)
    assert scan_calls(lib, scan(nseq=3), seq=FAKE) == (ssd.SSD_ERR_SEQIDX_BATCH,) * 2
    assert scan_calls(lib, scan(batch=1, nseq=4097), seq=FAKE) == (ssd.SSD_ERR_BAD_SHAPE,) * 2
    # z's strides play no part without z
    assert scan_calls(lib, scan(z_token_stride=-1), ws_bytes=0)[1] == ssd.SSD_ERR_WORKSPACE
    for name, k in (("ssd_scan_workspace_bytes", 0), ("ssd_scan_backward_workspace_bytes", 1)):
        size = ctypes.c_size_t(0)
        assert getattr(lib, name)(ctypes.byref(scan()), ctypes.byref(size)) == ssd.SSD_OK and size.value > 0
        assert scan_calls(lib, scan(), ws_bytes=size.value - 1)[k] == ssd.SSD_ERR_WORKSPACE
        assert scan_calls(lib, scan(), ws=None)[k] == ssd.SSD_ERR_WORKSPACE
        assert scan_calls(lib, scan(), ws=FAKE + 4)[k] == dims

    def step(p, state=FAKE, x=FAKE):
        return lib.ssd_scan_step(ctypes.byref(p), x, FAKE, FAKE, FAKE, FAKE, None, None, None, state, FAKE, None)

    assert step(scan(), state=FAKE + 4) == dims
    assert step(scan(seqlen=0, x_token_stride=-1), x=None) == null
    assert step(scan(dstate=8)) == dims


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), ssd.SSD_ERR_BAD_DTYPE), (dict(residual_dtype=2), ssd.SSD_ERR_BAD_DTYPE),
    (dict(dtype=F32, residual_dtype=BF16, out_dtype=F32), ssd.SSD_ERR_BAD_DTYPE),
    (dict(rows=0), ssd.SSD_ERR_BAD_SHAPE), (dict(channels=0), ssd.SSD_ERR_BAD_SHAPE),
    (dict(channels=32769), ssd.SSD_ERR_UNSUPPORTED_DIMS), (dict(eps=-1.0), ssd.SSD_ERR_BAD_OPTION),
    (dict(eps=float("nan")), ssd.SSD_ERR_BAD_OPTION), (dict(rows=1 << 40), ssd.SSD_ERR_TOO_LARGE)])
def test_norm_shapes(lib, kw, code):
    p = ctypes.byref(norm(**kw))
    size = ctypes.c_size_t(0)
    assert lib.ssd_add_norm(p, FAKE, FAKE, FAKE, FAKE, None, FAKE, None) == code
    assert lib.ssd_add_norm_backward(p, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == code
    assert lib.ssd_add_norm_backward_workspace_bytes(p, ctypes.byref(size)) == code


def test_norm_arguments(lib):
    null = ssd.SSD_ERR_NULL_ARG

    def fwd(p, x=FAKE, y=FAKE, scale=None):
        return lib.ssd_add_norm(ctypes.byref(p), x, None, None, y, scale, None, None)

    assert fwd(norm(), x=None) == null and fwd(norm(), y=None) == null
    assert fwd(norm(out_dtype=ssd.SSD_DTYPE_I8)) == null             # no place for the scales
    assert fwd(norm(out_dtype=F32)) == ssd.SSD_ERR_BAD_DTYPE         # y has x's dtype
    assert fwd(norm(out_dtype=9)) == ssd.SSD_ERR_BAD_DTYPE

    def back(dy=FAKE, dx=FAKE, dres=FAKE, ws=FAKE, n=1 << 40):
        return lib.ssd_add_norm_backward(ctypes.byref(norm()), dy, FAKE, None, None, dx, dres, FAKE, ws, n, None)

    size = ctypes.c_size_t(0)
    assert lib.ssd_add_norm_backward_workspace_bytes(ctypes.byref(norm()), ctypes.byref(size)) == ssd.SSD_OK
    assert back(dy=None) == null and back(dx=None, dres=None) == null
    assert back(n=size.value - 1) == ssd.SSD_ERR_WORKSPACE and back(ws=None) == ssd.SSD_ERR_WORKSPACE
    assert back(ws=FAKE + 4) == ssd.SSD_ERR_UNSUPPORTED_DIMS
    assert lib.ssd_add_norm_backward_workspace_bytes(ctypes.byref(norm()), None) == null


def test_tensors_on_the_cpu_are_refused():
    x, w, s = torch.zeros(1, 4, 8), torch.zeros(8, 4), torch.zeros(1, 4, 1, 16)
    for call in (lambda: ssd.conv_forward(x, w), lambda: ssd.conv_backward(x, w, x),
                 lambda: ssd.conv_step(x[0], w, torch.zeros(4, 3, 8)),
                 lambda: ssd.scan_forward(x, x, torch.zeros(8, 16), s, s),
                 lambda: ssd.scan_backward(x, x, torch.zeros(8, 16), s, s, x),
                 lambda: ssd.scan_step(x[0], x[0], torch.zeros(8, 16), s[0], s[0], torch.zeros(4, 8, 16)),
                 lambda: ssd.add_norm(x), lambda: ssd.add_norm_q8(x), lambda: ssd.add_norm_backward(x, x)):
        with pytest.raises(ValueError):
            call()
