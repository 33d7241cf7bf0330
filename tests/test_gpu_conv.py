"""The short convolution on the GPU against its float64 definition: outputs,
states and gradients over channel counts, lengths, widths, parts, strides and
packed rows; single tokens; refusals; streams and capture."""
import math

import pytest
import torch

from oracle import mixer
from tests.mixer_harness import DTYPES, Draw, announce, check, same, seq_idx_of, ssd, streams_and_graphs
from tests.test_gpu_parity import _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs(b, T, C, W, dtype, units, init, sliced, seed=3, bias=True):
    n, t = Draw(seed), DTYPES[dtype]
    x = n(b, T, 2 * C + 3, dtype=t)[..., 3:3 + C] if sliced else n(b, T, C, dtype=t)
    return {"x": x, "weight": n(C, W, scale=1 / math.sqrt(W)), "bias": n(C) if bias else None,
            "initial_states": n(units, W - 1, C, dtype=t) if init else None}


def both(b, T, C, W, dtype, init=False, sliced=False, split=None, starts=None, silu=True, bias=True, grad=True):
    announce("conv b%d T%d C%d W%d %s init %s sliced %s split %s starts %s" % (
        b, T, C, W, dtype, init, sliced, split, starts and starts[:6]))
    spans = mixer.packed(starts) if starts else mixer.rows(b, T)
    i = inputs(b, T, C, W, dtype, len(spans), init, sliced, bias=bias)
    packed = {"seq_idx": seq_idx_of(starts), "nseq": len(spans)} if starts else {}
    y, final = ssd.conv_forward(**i, silu=silu, split=split, **packed)
    want_y, want_final = mixer.conv_forward(i["x"], i["weight"], i["bias"], silu, i["initial_states"], spans)
    if split:
        assert all(p.is_contiguous() and p.shape[-1] == k for p, k in zip(y, split))
        y = torch.cat(y, -1)
    check("y", y, want_y)
    assert torch.equal(final.cpu().double(), want_final)     # inputs as they are
    if not grad:
        return
    n = Draw(4)
    dy, df = n(b, T, C, dtype=i["x"].dtype), n(len(spans), W - 1, C, dtype=i["x"].dtype) if init else None
    given = [p.contiguous() for p in torch.split(dy, split, -1)] if split else dy
    g = ssd.conv_backward(i["x"], i["weight"], given, bias=i["bias"], silu=silu,
                          initial_states=i["initial_states"], dfinal_states=df, **packed)
    want = mixer.conv_backward(i["x"], i["weight"], i["bias"], silu, i["initial_states"], spans, dy, df)
    assert (g["dbias"] is None) == (not bias)
    for k in g:
        if g[k] is not None:
            check(k, g[k], want[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,T,C,W,init,sliced", [
    (1, 1, 1, 4, False, False), (1, 1, 4, 2, True, False), (2, 2, 5, 4, True, True), (3, 3, 3, 3, False, False),
    (1, 4, 257, 4, True, False), (2, 5, 64, 2, False, True), (1, 67, 255, 3, True, False), (2, 130, 260, 4, True, True),
    (1, 515, 96, 4, False, False), (5, 33, 1028, 4, True, False), (1, 2, 7, 4, True, False)])
def test_rows(b, T, C, W, init, sliced, dtype):
    both(b, T, C, W, dtype, init, sliced)


@pytest.mark.parametrize("split", [(2, 1, 4), (5, 9), (256, 4, 4), (300, 17, 255)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts(split, dtype):
    both(2, 70, sum(split), 4, dtype, True, True, split)


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("init", [False, True])
@pytest.mark.parametrize("starts", [[0, 1], [0, 1, 2, 3, 4, 5], [0, 3, 4, 6, 16, 17, 31, 64, 65, 130, 131, 133],
                                    [0, 255, 256, 258, 400], [0, 127, 128, 129]])
def test_packed_rows(starts, init, W):
    both(1, starts[-1], 68, W, "f32", init, starts=starts)


def test_packed_rows_with_parts_bf16():
    both(1, 3001, 516, 4, "bf16", True, True, (500, 8, 8), [0, 2, 700, 701, 704, 2999, 3001])


def test_without_silu_and_bias():
    both(2, 40, 12, 4, "f32", True, silu=False, bias=False)
    both(2, 40, 12, 4, "bf16", silu=True, bias=False)


def test_long_strips():
    # enough tokens that a strip takes its longest length in both directions
    both(2, 9000, 1284, 4, "bf16", True, grad=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,C,W,sliced", [(1, 1, 4, False), (3, 7, 3, True), (2, 1792, 4, True), (5, 260, 2, False)])
def test_steps_continue_the_forward(b, C, W, sliced, dtype):
    announce("conv steps b%d C%d W%d %s" % (b, C, W, dtype))
    i = inputs(b, 9, C, W, dtype, b, True, sliced)
    y, final = ssd.conv_forward(**i)
    head = {**i, "x": i["x"][:, :4]}
    y0, state = ssd.conv_forward(**head)
    rest = [ssd.conv_step(i["x"][:, t], i["weight"], state, bias=i["bias"]) for t in range(4, 9)]
    assert same(torch.cat([y0, torch.stack(rest, 1)], 1), y) and same(state, final)


def test_an_infinite_sequence_stays_by_itself():
    announce("conv: infinities and NaN of one packed sequence")
    starts = [0, 5, 9, 40]
    i = inputs(1, 40, 20, 4, "f32", 3, True, False)
    seq = {"seq_idx": seq_idx_of(starts), "nseq": 3}
    dy = Draw(9)(1, 40, 20)
    clean = ssd.conv_forward(**i, **seq)[0], ssd.conv_backward(i["x"], i["weight"], dy, bias=i["bias"], **seq,
                                                             initial_states=i["initial_states"])["dx"]
    i["x"][0, 5:9] = float("inf")
    i["x"][0, 7] = float("nan")
    i["initial_states"][1] = float("-inf")
    got = ssd.conv_forward(**i, **seq)[0], ssd.conv_backward(i["x"], i["weight"], dy, bias=i["bias"], **seq,
                                                             initial_states=i["initial_states"])["dx"]
    for a, c in zip(got, clean):
        assert same(a[:, :5], c[:, :5]) and same(a[:, 9:], c[:, 9:])


def test_extreme_preactivations():
    """SiLU at both ends: no NaN from an exponential that overflows."""
    announce("conv: SiLU of large values")
    v = torch.tensor([-3e38, -1e4, -104.5, -90.0, -88.0, -20.0, 0.0, 20.0, 88.0, 1e4, 3e38]).cuda().view(1, 1, -1)
    w = torch.zeros(11, 2).cuda()
    w[:, 1] = 1.0
    y, _ = ssd.conv_forward(v, w)
    want, _ = mixer.conv_forward(v, w, None, True, None, mixer.rows(1, 1))
    # a sigmoid below 2^-126 (v < -87.3) may count as 0
    v = v.cpu().double()
    lost = torch.where((v < -87.3) & (v > -105), v.abs() * 2.0 ** -126, 0.0)
    assert torch.all((y.cpu().double() - want).abs() <= 8 * 2.0 ** -24 * want.abs() + lost)


def test_refusals():
    announce("conv refusals")
    i = inputs(2, 6, 8, 4, "f32", 2, True, False)
    dy, state = Draw(5)(2, 6, 8), i["initial_states"].clone()
    seq = torch.zeros(1, 6, dtype=torch.int32).cuda()

    def refuse(error, call, **change):
        with pytest.raises(error):
            call(**{**i, **change})

    f, back = ssd.conv_forward, lambda **k: ssd.conv_backward(dy=k.pop("dy", dy), **k)
    for call in (f, back):
        refuse(TypeError, call, x=i["x"].half())
        refuse(ValueError, call, x=i["x"].cpu())
        refuse(ValueError, call, x=i["x"].transpose(1, 2).contiguous().transpose(1, 2))
        refuse(ValueError, call, x=i["x"][0])
        refuse(TypeError, call, weight=i["weight"].bfloat16())
        refuse(ValueError, call, weight=i["weight"][:4])
        refuse(ValueError, call, weight=i["weight"].t().contiguous().t())
        refuse(ValueError, call, bias=i["bias"].cpu())
        refuse(TypeError, call, initial_states=state.bfloat16())
        refuse(ValueError, call, initial_states=state[:1])
        refuse(ValueError, call, seq_idx=seq, nseq=1)                       # a packed row is one row
        refuse(ssd.SsdError, call, weight=Draw(1)(8, 5), initial_states=None)   # width 5
        refuse(ssd.SsdError, call, weight=Draw(1)(8, 1), initial_states=None)
    one = {**i, "x": i["x"][:1], "initial_states": None}
    for bad in (0, 7):
        with pytest.raises(ValueError):
            f(**one, seq_idx=seq, nseq=bad)
    with pytest.raises(TypeError):
        f(**one, seq_idx=seq.long(), nseq=1)
    with pytest.raises(ValueError):
        f(**i, split=(4, 5))
    with pytest.raises(ValueError):
        f(**i, split=(2, 2, 2, 2))
    with pytest.raises(ValueError):
        f(**i, split=(8, 0))
    with pytest.raises(ValueError):
        f(**i, out=torch.empty(2, 6, 9).cuda())
    with pytest.raises(ssd.SsdError) as e:
        f(**{**i, "x": i["x"][:, :0]})
    assert e.value.code == ssd.SSD_ERR_BAD_SHAPE
    refuse(ValueError, back, dy=dy[:, :5])
    refuse(ValueError, back, workspace=torch.empty(16, dtype=torch.uint8).cuda())
    with pytest.raises(ValueError):
        ssd.conv_step(i["x"], i["weight"], state)
    with pytest.raises(ValueError):
        ssd.conv_step(i["x"][:, 0], i["weight"], state[:, :2])
    with pytest.raises(TypeError):
        ssd.conv_step(i["x"][:, 0], i["weight"], state.bfloat16())


def test_streams_and_capture():
    announce("conv on a side stream and captured")
    i = inputs(2, 50, 40, 4, "bf16", 2, True, True)
    dy, start, state = Draw(6)(2, 50, 40).bfloat16(), i["initial_states"], i["initial_states"].clone()
    streams_and_graphs(lambda: ssd.conv_forward(**i))
    streams_and_graphs(lambda: ssd.conv_backward(i["x"], i["weight"], dy, bias=i["bias"]))
    streams_and_graphs(lambda: (ssd.conv_step(i["x"][:, 0], i["weight"], state), state), lambda: state.copy_(start))
