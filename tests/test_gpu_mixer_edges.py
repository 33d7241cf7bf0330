"""The operators around the layer at the ends of their ranges on the GPU, against
their float64 definitions: SiLU where its exponential overflows."""
import pytest
import torch

from oracle import mixer
from tests.mixer_harness import DTYPES, Draw, announce, check, same, seq_idx_of, ssd
from tests.test_gpu_parity import _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def large_negatives(dtype):
    """From -110 to -80: every bf16 value; 30,001 float32 ones, 0.001 apart."""
    if dtype == "f32":
        return torch.linspace(-110, -80, 30001)
    return torch.arange(-110, -79.75, 0.25).bfloat16().unique()


def lost(v):
    """What v sigmoid(v) and its derivative may be off in all: a sigmoid below 2^-126 (v <
    -87.3) may count as 0."""
    v = v.double()
    return torch.where(v < -87.3, v.abs() * 2.0 ** -126, 0.0)


def near(name, got, want, roundings, apart):
    """Every value within so many roundings of its own, and of its type's one."""
    assert got.shape == want.shape
    got = got.detach()
    share = roundings * 2.0 ** -24 + (2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0)
    err = (got.cpu().double() - want).abs()
    bad = ~(err <= share * want.abs() + apart)   # (a NaN is bad)
    assert not bad.any(), "%s: %d of %d, first %s, want %s" % (name, bad.sum(), bad.numel(), got[bad.to(got.device)][0], want[bad][0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_convolution_of_large_negative_sums(dtype):
    """Exponentials, reciprocal, products: fewer than 16 roundings."""
    v = large_negatives(dtype)
    announce("conv: SiLU of %d values from -110 to -80 %s" % (len(v), dtype))
    n, apart = len(v), lost(v)
    x, w = v.cuda().view(1, 1, n), torch.zeros(n, 2).cuda()
    w[:, 1] = 1.0
    want, _ = mixer.conv_forward(x, w, None, True, None, mixer.rows(1, 1))
    near("y", ssd.conv_forward(x, w)[0], want, 16, apart)
    near("step", ssd.conv_step(x[0], w, torch.zeros(1, 1, n, dtype=x.dtype).cuda()), want[0], 16, apart)
    dy, bias = torch.ones_like(x), torch.zeros(n).cuda()
    g = ssd.conv_backward(x, w, dy, bias=bias)
    want = mixer.conv_backward(x, w, bias, True, None, mixer.rows(1, 1), dy, None)
    near("dx", g["dx"], want["dx"], 16, apart)
    near("dbias", g["dbias"], want["dbias"], 16, apart)
    near("dweight", g["dweight"], want["dweight"], 16, (apart * 110)[:, None])
    assert torch.all(g["dinit"] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_gated_by_large_negatives(dtype):
    """One token a channel, all operands 1: a value is a sum of at most 33 products with
    one SiLU (or a derivative), no larger than 64 of it, all of one sign: 64 roundings;
    the sums over channels are of 64 lanes and of up to 469 tiles."""
    v = large_negatives(dtype)
    announce("scan: a gate of %d values from -110 to -80 %s" % (len(v), dtype))
    E, N, apart = len(v), 16, 64 * lost(v)
    t = DTYPES[dtype]
    one = torch.ones(1, 1, E, dtype=t).cuda()
    i = {"x": one, "dt": one, "A_log": torch.zeros(E, N).cuda(), "B": torch.ones(1, 1, 1, N, dtype=t).cuda(),
         "C": torch.ones(1, 1, 1, N, dtype=t).cuda(), "D": torch.ones(E).cuda(), "z": v.cuda().view(1, 1, E)}
    state = torch.ones(1, E, N).cuda()
    names = {**i, "dt_bias": None, "softplus": False, "init": state, "spans": mixer.rows(1, 1)}
    want, want_f = mixer.scan_forward(**names)
    y, f = ssd.scan_forward(**i, dt_softplus=False, initial_states=state)
    near("y", y, want, 64, apart)
    near("final", f, want_f, 64, 0.0)
    g = ssd.scan_backward(**i, dy=one, dt_softplus=False, initial_states=state)
    want_g = mixer.scan_backward(**names, dy=one, dfinal=None)
    for k in ("dx", "ddt", "dz", "dD"):
        near(k, g[k], want_g[k], 64, apart)
    for k in ("dA_log", "dinit"):
        near(k, g[k], want_g[k], 64, apart[:, None])
    for k in ("dB", "dC"):
        near(k, g[k], want_g[k], 64 + 64 + 469, apart.sum())
    step = ssd.scan_step(one[:, 0], one[:, 0], i["A_log"], i["B"][:, 0], i["C"][:, 0], state, D=i["D"], z=i["z"][:, 0],
                         dt_softplus=False)
    near("step", step, want[0], 64, apart)


def packed_scan(T, starts, softplus=True, seed=3):
    n = Draw(seed)
    E, N, units = 20, 16, len(starts) - 1
    i = {"x": n(1, T, E), "dt": n(1, T, E, scale=0.7), "A_log": n(E, N, scale=0.3), "B": n(1, T, 1, N), "C": n(1, T, 1, N),
         "D": n(E), "z": n(1, T, E), "dt_bias": n(E) if softplus else None, "dt_softplus": softplus,
         "initial_states": n(units, E, N), "seq_idx": seq_idx_of(starts), "nseq": units}
    return i, {"dy": n(1, T, E), "dfinal_states": n(units, E, N)}


@pytest.mark.parametrize("what", [("dt",), ("z", "B", "C"), ("dy", "dfinal_states"), ("x", "dt", "z", "B", "C", "dy")])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("T,starts", [(40, [0, 5, 9, 40]), (700, [0, 130, 300, 700])])
def test_an_odd_sequence_of_the_scan_stays_by_itself(T, starts, value, what):
    """Whatever one packed sequence holds, the others' results keep their bits."""
    announce("scan: %s in %s of one packed sequence of %d tokens" % (value, what, T))
    i, back = packed_scan(T, starts)

    def results():
        y, f = ssd.scan_forward(**i)
        g = ssd.scan_backward(**i, **back)
        return [y, g["dx"], g["ddt"], g["dz"], g["dB"], g["dC"]], [f, g["dinit"]]

    clean = results()
    for k in what:
        t = {**i, **back}[k]
        if k == "dfinal_states":
            t[1] = value
        else:
            t[:, starts[1]:starts[2]] = value
    got = results()
    for a, c in zip(got[0], clean[0]):
        assert same(a[:, :starts[1]], c[:, :starts[1]]) and same(a[:, starts[2]:], c[:, starts[2]:])
    for a, c in zip(got[1], clean[1]):
        assert same(a[[0, 2]], c[[0, 2]])


def test_packed_sequences_that_grow():
    """Without softplus time steps may be negative and states grow: each of the eleven
    sequences by up to 2^70 here, which the others do not meet.  (An exponent of 17 is off
    by 17 roundings, four tokens' by 70: within what check allows.)"""
    announce("scan: packed sequences with negative time steps")
    starts = [0, 4, *range(6, 40, 4), 40]     # (tiles of 8 tokens start within sequences)
    i, back = packed_scan(40, starts, softplus=False)
    i["dt"].fill_(-0.75)
    i["A_log"].copy_(torch.log(torch.arange(1, 17).float()).expand(20, 16))
    spans = mixer.packed(starts)
    names = {"softplus": False, "init": i["initial_states"], "spans": spans,
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C", "D", "z", "dt_bias")}}
    y, f = ssd.scan_forward(**i)
    want_y, want_f = mixer.scan_forward(**names)
    check("y", y, want_y)
    check("final", f, want_f)
    g = ssd.scan_backward(**i, **back)
    want = mixer.scan_backward(**names, dy=back["dy"], dfinal=back["dfinal_states"])
    for k in ("dx", "ddt", "dz", "dB", "dC", "dA_log", "dD", "dinit"):
        check(k, g[k], want[k])


def test_decay_rates_of_any_size():
    """A = -exp(A_log) beyond float32 (the state is forgotten, by any time step but 0) and
    0 (nothing is): no NaN where the definition has none."""
    announce("scan: A_log from -inf to 1e30")
    a_log = torch.tensor([float("-inf"), -1e30, -200.0, -104.0, -95.0, 0.0, 1.0, 80.0, 87.0, 88.5, 89.0, 90.0, 93.0, 95.0,
                          97.0, 104.0, 300.0, 700.0])
    n, E, T = Draw(7), len(a_log), 40
    i = {"x": n(2, T, E), "dt": n(2, T, E).abs() + 0.01, "A_log": a_log.cuda()[:, None].repeat(1, 16), "B": n(2, T, 1, 16),
         "C": n(2, T, 1, 16), "initial_states": n(2, E, 16)}
    i["dt"][:, ::3] = 0.0
    names = {"D": None, "z": None, "dt_bias": None, "softplus": False, "init": i["initial_states"], "spans": mixer.rows(2, T),
             **{k: i[k] for k in ("x", "dt", "A_log", "B", "C")}}
    y, f = ssd.scan_forward(**i, dt_softplus=False)
    want_y, want_f = mixer.scan_forward(**names)
    check("y", y, want_y)
    check("final", f, want_f)
    dy, df = n(2, T, E), n(2, E, 16)
    g, want = ssd.scan_backward(**i, dy=dy, dfinal_states=df, dt_softplus=False), mixer.scan_backward(**names, dy=dy, dfinal=df)
    for k in ("dx", "dB", "dC", "dinit"):
        check(k, g[k], want[k])
    for e, a in enumerate(a_log.tolist()):   # 
        # ddt holds A itself at the time steps of 0, times up to 10 here: at A_log 87 (A
        # 6.1e37) the definition's largest is 6.3e38, more than float32 holds (3.4e38)
        if a <= 80:
            check("ddt of A_log %g" % a, g["ddt"][..., e], want["ddt"][..., e])
        if 2 < a:
            assert torch.all(g["dA_log"][e] == 0), a
        elif a > -87:
            check("dA_log of %g" % a, g["dA_log"][e], want["dA_log"][e])
        else:                                # (A itself is below 2^-126 and may count as 0)
            assert torch.all(g["dA_log"][e].cpu().double().abs() <= 2 * want["dA_log"][e].abs() + 2.0 ** -126), a
    state = i["initial_states"].clone()
    for t in range(4):
        step = ssd.scan_step(i["x"][:, t], i["dt"][:, t], i["A_log"], i["B"][:, t], i["C"][:, t], state, dt_softplus=False)
        check("step", step, want_y[:, t])


def test_a_decay_rate_that_is_no_number():
    """A NaN in A_log is a NaN in its channel's results, and in no other's."""
    announce("scan: NaN in A_log")
    n, E, T = Draw(7), 70, 300
    i = {"x": n(1, T, E), "dt": n(1, T, E), "A_log": n(E, 16), "B": n(1, T, 1, 16), "C": n(1, T, 1, 16)}
    dy = n(1, T, E)
    state = torch.zeros(1, E, 16).cuda()

    def results():
        y, f = ssd.scan_forward(**i)
        g = ssd.scan_backward(**i, dy=dy)
        s = state.clone()
        step = ssd.scan_step(i["x"][:, 0], i["dt"][:, 0], i["A_log"], i["B"][:, 0], i["C"][:, 0], s)
        return {"y": y, "dx": g["dx"], "ddt": g["ddt"], "step": step}, {"f": f, "dA_log": g["dA_log"][None], "s": s}

    clean = results()
    i["A_log"][3, 5] = float("nan")
    got = results()
    others = [e for e in range(E) if e != 3]
    for k, t in got[0].items():
        assert same(t[..., others], clean[0][k][..., others]), k
    for k in ("y", "ddt", "step"):
        assert torch.isnan(got[0][k][..., 3]).all(), k
    for k, t in got[1].items():
        assert same(t[:, others], clean[1][k][:, others]), k
        assert torch.isnan(t[:, 3, 5]).all(), k


@pytest.mark.parametrize("to", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("C", [8, 300, 9000])
def test_rows_of_zeros_without_eps(C, to):
    announce("add_norm_q8: rows of zeros, eps 0, %d channels" % C)
    x = Draw(2)(4, C)
    x[1] = 0.0
    weight = torch.ones(C).cuda()
    q, scale, _ = ssd.add_norm_q8(x, weight, eps=0.0, dtype=to)
    assert scale[1] == 0 and torch.all(q[1].float() == 0)
    want, _ = mixer.add_norm(x[[0, 2, 3]], weight, None, 0.0)
    check("scale", scale[[0, 2, 3]], want.abs().amax(-1) / (127.0 if to is torch.int8 else 448.0))
    weight.zero_()                       # (and t = r w of rows that are not)
    q, scale, _ = ssd.add_norm_q8(x, weight, eps=0.0, dtype=to)
    assert torch.all(scale == 0) and torch.all(q.float() == 0)
