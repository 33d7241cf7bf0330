"""The selective scan on the GPU against its float64 definition: outputs, states
and gradients over channel and state counts, groups, lengths (one chunk and many),
packed rows, strides and missing operands; single tokens; refusals; streams and
capture."""
import pytest
import torch

from oracle import mixer
from tests.mixer_harness import DTYPES, Draw, announce, check, same, seq_idx_of, ssd, streams_and_graphs
from tests.test_gpu_parity import _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs(b, T, E, N, G, dtype, units, gate=True, init=True, D=True, bias=True, softplus=True, sliced=False, seed=3):
    n, t = Draw(seed), DTYPES[dtype]

    def act(*shape, scale=1.0, pad=2):
        if not sliced:
            return n(*shape, dtype=t, scale=scale)
        wide = n(*shape[:-1], shape[-1] + 2 * pad, dtype=t, scale=scale)
        return wide[..., pad:pad + shape[-1]]

    def bc():   # slices of a wider projection: batch, token, then groups and states
        if not sliced:
            return n(b, T, G, N, dtype=t)
        return n(b, T, G * N + 6, dtype=t)[..., 4:4 + G * N].unflatten(-1, (G, N))

    dt = act(b, T, E, scale=0.7)
    if not softplus:
        dt = dt.abs()
    return {"x": act(b, T, E, pad=3), "dt": dt, "A_log": torch.log(torch.arange(1, N + 1).float()).cuda() + n(E, N, scale=.1),
            "B": bc(), "C": bc(), "D": n(E) if D else None, "z": act(b, T, E, pad=1) if gate else None,
            "dt_bias": n(E) - 3 if bias and softplus else n(E).abs() if bias else None, "dt_softplus": softplus,
            "initial_states": n(units, E, N) if init else None}


def both(b, T, E, N=16, G=1, dtype="f32", starts=None, grad=True, **more):
    announce("scan b%d T%d E%d N%d G%d %s starts %s %s" % (b, T, E, N, G, dtype, starts and starts[:6], more))
    spans = mixer.packed(starts) if starts else mixer.rows(b, T)
    i = inputs(b, T, E, N, G, dtype, len(spans), **more)
    packed = {"seq_idx": seq_idx_of(starts), "nseq": len(spans)} if starts else {}
    y, final = ssd.scan_forward(**i, **packed)
    names = {"softplus": i["dt_softplus"], "init": i["initial_states"], "spans": spans,
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C", "D", "z", "dt_bias")}}
    want_y, want_final = mixer.scan_forward(**names)
    check("y", y, want_y)
    check("final", final, want_final)
    if not grad:
        return
    n = Draw(4)
    dy = n(b, T, E, dtype=i["x"].dtype)
    df = n(len(spans), E, N) if i["initial_states"] is not None else None
    g = ssd.scan_backward(**i, dy=dy, dfinal_states=df, **packed)
    want = mixer.scan_backward(**names, dy=dy, dfinal=df)
    for name, given in (("dz", i["z"]), ("dD", i["D"]), ("ddt_bias", i["dt_bias"])):
        assert (g[name] is None) == (given is None)
    for k in g:
        if g[k] is not None:
            check(k, g[k], want[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,T,E,N,G", [
    (1, 1, 1, 16, 1), (2, 1, 65, 16, 1), (1, 7, 64, 16, 1), (3, 8, 5, 32, 1), (2, 9, 130, 16, 2), (1, 15, 63, 48, 3),
    (1, 16, 66, 16, 1), (2, 17, 200, 16, 8), (1, 33, 64, 256, 1), (2, 130, 70, 16, 1), (1, 200, 129, 64, 1)])
def test_rows(b, T, E, N, G, dtype):
    both(b, T, E, N, G, dtype)


@pytest.mark.parametrize("T", [127, 128, 129, 191, 640, 1000])
def test_chunk_edges(T):
    both(1, T, 65, 16)


@pytest.mark.parametrize("b,T,E,N,G", [(4, 300, 768, 16, 1), (1, 2000, 80, 32, 2), (1, 300, 64, 128, 1)])
def test_many_chunks_bf16(b, T, E, N, G):
    both(b, T, E, N, G, "bf16")


@pytest.mark.parametrize("init", [False, True])
@pytest.mark.parametrize("starts", [[0, 1], [0, 1, 2, 3, 4, 5], [0, 3, 4, 16, 17, 31, 64, 65, 130, 131, 133],
                                    [0, 64, 128, 129, 192, 255, 256, 300], [0, 1, 500, 501, 700]])
def test_packed_rows(starts, init):
    both(1, starts[-1], 66, 16, 1, "f32", starts, init=init)


def test_packed_rows_bf16():
    both(1, 900, 130, 32, 2, "bf16", [0, 2, 300, 301, 304, 880, 900])


@pytest.mark.parametrize("more", [{"gate": False}, {"D": False}, {"bias": False}, {"softplus": False},
                                  {"softplus": False, "bias": False, "gate": False, "D": False, "init": False},
                                  {"init": False}])
def test_missing_operands(more):
    both(2, 150, 70, 16, **more)
    both(2, 20, 70, 32, 2, "bf16", **more)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slices(dtype):
    both(2, 150, 70, 32, 2, dtype, sliced=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,E,N,G,sliced", [(1, 1, 16, 1, False), (3, 70, 48, 2, True), (2, 1536, 16, 1, True), (2, 9, 256, 1, False)])
def test_steps_continue_the_forward(b, E, N, G, sliced, dtype):
    announce("scan steps b%d E%d N%d G%d %s" % (b, E, N, G, dtype))
    i = inputs(b, 9, E, N, G, dtype, b, sliced=sliced)
    names = {"softplus": True, "init": i["initial_states"], "spans": mixer.rows(b, 9),
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C", "D", "z", "dt_bias")}}
    want_y, want_final = mixer.scan_forward(**names)
    head = {k: v[:, :4] if k in ("x", "dt", "z", "B", "C") else v for k, v in i.items()}
    y0, state = ssd.scan_forward(**head)
    rest = [ssd.scan_step(i["x"][:, t], i["dt"][:, t], i["A_log"], i["B"][:, t], i["C"][:, t], state, D=i["D"],
                          z=i["z"][:, t], dt_bias=i["dt_bias"]) for t in range(4, 9)]
    check("y", torch.cat([y0, torch.stack(rest, 1)], 1), want_y)
    check("state", state, want_final)


@pytest.mark.parametrize("T,starts", [(40, [0, 5, 9, 40]), (700, [0, 130, 300, 700])])
def test_an_infinite_sequence_stays_by_itself(T, starts):
    announce("scan: infinities and NaN of one packed sequence")
    i = inputs(1, T, 20, 16, 1, "f32", 3)
    seq = {"seq_idx": seq_idx_of(starts), "nseq": 3}
    n = Draw(9)
    dy, df = n(1, T, 20), n(3, 20, 16)

    def results():
        y, f = ssd.scan_forward(**i, **seq)
        g = ssd.scan_backward(**i, dy=dy, dfinal_states=df, **seq)
        return [y, g["dx"], g["ddt"], g["dz"], g["dB"], g["dC"]], [f, g["dinit"]]

    clean = results()
    i["x"][0, starts[1]:starts[2]] = float("inf")
    i["x"][0, starts[1] + 1] = float("nan")
    i["initial_states"][1] = float("nan")
    got = results()
    for a, c in zip(got[0], clean[0]):
        assert same(a[:, :starts[1]], c[:, :starts[1]]) and same(a[:, starts[2]:], c[:, starts[2]:])
    for a, c in zip(got[1], clean[1]):
        assert same(a[[0, 2]], c[[0, 2]])


@pytest.mark.parametrize("E", [5, 64])
def test_an_infinite_operand_makes_no_nan_of_its_own(E):
    """One channel's input is infinite at one token: the sums over channels are
    infinite where the definition's are, and a NaN only where they are."""
    announce("scan: one infinite operand (%d channels)" % E)
    i = inputs(1, 40, E, 16, 1, "f32", 1, gate=False, init=False)
    i["x"][0, 11, E - 1] = float("inf")
    dy = Draw(9)(1, 40, E)
    g = ssd.scan_backward(**i, dy=dy)
    names = {"softplus": True, "init": None, "spans": mixer.rows(1, 40),
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C", "D", "z", "dt_bias")}}
    want = mixer.scan_backward(**names, dy=dy, dfinal=None)
    for k in ("dB", "dC"):
        got = g[k].cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want[k])) and torch.equal(torch.isinf(got), torch.isinf(want[k]))


def test_strides_that_play_no_part():
    """Strides over a single batch row or token may be anything."""
    announce("scan, conv: strides over one row or token")
    i = inputs(1, 9, 70, 16, 1, "bf16", 1)
    want = ssd.scan_forward(**i)
    odd = {**i, "B": i["B"].as_strided((1, 9, 1, 16), (7, 16, 16, 1)), "C": i["C"].as_strided((1, 9, 1, 16), (13, 16, 5, 1)),
           "x": i["x"].as_strided((1, 9, 70), (1, 70, 1))}
    assert same(ssd.scan_forward(**odd), want)
    one = {k: v[:, :1] if k in ("x", "dt", "z", "B", "C") else v for k, v in i.items()}
    want = ssd.scan_forward(**one)
    odd = {**one, "B": one["B"].as_strided((1, 1, 1, 16), (7, 3, 1, 1)), "x": one["x"].as_strided((1, 1, 70), (3, 1 << 40, 1))}
    assert same(ssd.scan_forward(**odd), want)
    w = Draw(1)(70, 4)
    assert same(ssd.conv_forward(odd["x"], w), ssd.conv_forward(one["x"], w))


def test_small_and_large_steps():
    """dt over its whole range: softplus to float32's precision (2e-7 relative) where
    it is as small as e^v and where it is v, seen through one token."""
    announce("scan: softplus")
    v = torch.cat([torch.linspace(-80, 80, 1601), torch.tensor([-1e4, 1e4])]).cuda()
    E = v.numel()
    one = torch.ones(1, 1, E).cuda()
    A_log = torch.zeros(E, 16).cuda()
    B = torch.ones(1, 1, 1, 16).cuda()
    _, final = ssd.scan_forward(one, v.view(1, 1, E), A_log, B, B)
    want = torch.logaddexp(v.cpu().double(), torch.zeros(E, dtype=torch.float64))
    err = (final[0, :, 0].cpu().double() - want).abs()
    assert torch.all(err <= 8 * 2.0 ** -24 * want)


def test_decays_that_vanish():
    """Decays far below the float32 range: the state is what the last token put in."""
    announce("scan: vanishing decays")
    both(1, 300, 66, 16, dtype="f32", seed=3)
    i = inputs(1, 300, 66, 16, 1, "f32", 1)
    i["dt"] = i["dt"].abs() * 200
    names = {"softplus": True, "init": i["initial_states"], "spans": mixer.rows(1, 300),
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C", "D", "z", "dt_bias")}}
    y, final = ssd.scan_forward(**i)
    want_y, want_final = mixer.scan_forward(**names)
    check("y", y, want_y)
    check("final", final, want_final)
    dy = Draw(4)(1, 300, 66)
    g, want = ssd.scan_backward(**i, dy=dy), mixer.scan_backward(**names, dy=dy, dfinal=None)
    for k in ("dx", "ddt", "dB", "dC", "dz", "dD"):
        check(k, g[k], want[k])


def test_refusals():
    announce("scan refusals")
    i = inputs(2, 6, 8, 16, 2, "bf16", 2)
    dy = Draw(5)(2, 6, 8).bfloat16()
    f, back = ssd.scan_forward, lambda **k: ssd.scan_backward(dy=k.pop("dy", dy), **k)

    def refuse(error, call, **change):
        with pytest.raises(error) as e:
            call(**{**i, **change})
        return e.value

    odd = Draw(1)(2, 6, 2 * 16 + 1).bfloat16()[..., 1:].unflatten(-1, (2, 16))
    for call in (f, back):
        refuse(TypeError, call, x=i["x"].half())
        refuse(ValueError, call, x=i["x"].cpu())
        refuse(TypeError, call, dt=i["dt"].float())
        refuse(TypeError, call, z=i["z"].float())
        refuse(ValueError, call, z=i["z"][:1])
        refuse(TypeError, call, A_log=i["A_log"].bfloat16())
        refuse(ValueError, call, A_log=i["A_log"].t().contiguous().t())
        refuse(ValueError, call, D=i["D"].cpu())
        refuse(ValueError, call, B=i["B"].transpose(2, 3).contiguous().transpose(2, 3))
        refuse(ValueError, call, C=i["C"].transpose(1, 2).contiguous().transpose(1, 2)[..., :8])
        refuse(ValueError, call, initial_states=i["initial_states"][:1])
        refuse(ValueError, call, seq_idx=torch.zeros(1, 6, dtype=torch.int32).cuda(), nseq=1)
        assert refuse(ssd.SsdError, call, B=odd).code == ssd.SSD_ERR_UNSUPPORTED_DIMS    # 2-byte aligned
        n24 = {"A_log": Draw(1)(8, 24), "B": Draw(1)(2, 6, 2, 24).bfloat16(), "C": Draw(1)(2, 6, 2, 24).bfloat16()}
        assert refuse(ssd.SsdError, call, **n24, initial_states=None).code == ssd.SSD_ERR_UNSUPPORTED_DIMS
    with pytest.raises(ssd.SsdError) as e:
        f(**{k: v[:, :0] if k in ("x", "dt", "z", "B", "C") else v for k, v in i.items()})
    assert e.value.code == ssd.SSD_ERR_BAD_SHAPE
    refuse(ValueError, back, dy=dy[:, :5])
    refuse(TypeError, back, dy=dy.float())
    refuse(ValueError, back, workspace=torch.empty(16, dtype=torch.uint8).cuda())
    refuse(ValueError, f, out=torch.empty(2, 6, 9).cuda().bfloat16())
    state = i["initial_states"].clone()
    step = dict(x=i["x"][:, 0], dt=i["dt"][:, 0], A_log=i["A_log"], B=i["B"][:, 0], C=i["C"][:, 0], state=state)
    for bad, error in (({"state": state.bfloat16()}, TypeError), ({"state": state[:1]}, ValueError),
                       ({"B": i["B"][:, 0].float()}, TypeError), ({"x": i["x"]}, ValueError)):
        with pytest.raises(error):
            ssd.scan_step(**{**step, **bad})


def test_streams_and_capture():
    announce("scan on a side stream and captured")
    i = inputs(2, 300, 70, 32, 1, "bf16", 2)
    dy, start, state = Draw(6)(2, 300, 70).bfloat16(), i["initial_states"], i["initial_states"].clone()
    streams_and_graphs(lambda: ssd.scan_forward(**i))
    streams_and_graphs(lambda: ssd.scan_backward(**i, dy=dy))
    streams_and_graphs(lambda: (ssd.scan_step(i["x"][:, 0], i["dt"][:, 0], i["A_log"], i["B"][:, 0], i["C"][:, 0], state),
                                state), lambda: state.copy_(start))
