"""The definitions of ``oracle/mixer.py``: gradients against central differences,
states that carry a sequence over a cut, packed rows as separate sequences."""
import pytest
import torch

from oracle import mixer


def randn(*shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def differences(f, inputs, grads, outs):
    """d/de of sum(out . f(inputs + e direction)) against the gradients' products."""
    for k, (name, t) in enumerate(inputs.items()):
        way = randn(*t.shape, seed=100 + k)
        step = 1e-5

        def value(e):
            got = f(**{**inputs, name: t + e * way})
            return sum((a * b).sum() for a, b in zip(got, outs))

        slope = (value(step) - value(-step)) / (2 * step)
        # central differences: step^2 of the third derivative and 1e-16 / step of the value
        assert abs(slope - (grads[name] * way).sum()) <= 1e-6 * (1 + abs(slope)), name


SPANS = [mixer.rows(2, 5), mixer.packed([0, 1, 2, 5, 9, 10])]


@pytest.mark.parametrize("spans", SPANS)
@pytest.mark.parametrize("W,silu", [(2, True), (4, True), (3, False)])
def test_conv_gradients(W, silu, spans):
    b, T = max(r for r, _, _ in spans) + 1, max(hi for _, _, hi in spans)
    C, n = 3, len(spans)
    i = {"x": randn(b, T, C, seed=1), "weight": randn(C, W, seed=2), "bias": randn(C, seed=3),
         "init": randn(n, W - 1, C, seed=4)}
    dy, df = randn(b, T, C, seed=5), randn(n, W - 1, C, seed=6)
    g = mixer.conv_backward(i["x"], i["weight"], i["bias"], silu, i["init"], spans, dy, df)
    differences(lambda **k: mixer.conv_forward(silu=silu, spans=spans, **k), i,
                {"x": g["dx"], "weight": g["dweight"], "bias": g["dbias"], "init": g["dinit"]}, (dy, df))


@pytest.mark.parametrize("spans", SPANS)
@pytest.mark.parametrize("G,gate,softplus", [(1, True, True), (2, False, True), (2, True, False)])
def test_scan_gradients(G, gate, softplus, spans):
    b, T = max(r for r, _, _ in spans) + 1, max(hi for _, _, hi in spans)
    E, N, n = 4, 3, len(spans)
    i = {"x": randn(b, T, E, seed=1), "dt": randn(b, T, E, seed=2).abs(), "A_log": randn(E, N, seed=3),
         "B": randn(b, T, G, N, seed=4), "C": randn(b, T, G, N, seed=5), "D": randn(E, seed=6),
         "dt_bias": randn(E, seed=7).abs(), "init": randn(n, E, N, seed=8)}
    if gate:
        i["z"] = randn(b, T, E, seed=9)
    rest = {"softplus": softplus, "spans": spans, **({} if gate else {"z": None})}
    dy, df = randn(b, T, E, seed=10), randn(n, E, N, seed=11)
    g = mixer.scan_backward(dy=dy, dfinal=df, **i, **rest)
    differences(lambda **k: mixer.scan_forward(**k, **rest), i,
                {"init" if k == "dinit" else k[1:]: v for k, v in g.items()}, (dy, df))


def test_norm_gradients():
    i = {"x": randn(3, 7, seed=1), "residual": randn(3, 7, seed=2), "weight": randn(7, seed=3)}
    dy, dr = randn(3, 7, seed=4), randn(3, 7, seed=5)
    g = mixer.add_norm_backward(dy, i["x"] + i["residual"], i["weight"], dr, 1e-2)
    differences(lambda **k: mixer.add_norm(eps=1e-2, **k), i,
                {"x": g["dx"], "residual": g["dresidual"], "weight": g["dweight"]}, (dy, dr))


def test_states_carry_a_sequence_over_a_cut():
    x, w = randn(1, 9, 3, seed=1), randn(3, 4, seed=2)
    whole, end = mixer.conv_forward(x, w, None, True, None, mixer.rows(1, 9))
    for cut in (1, 2, 5):
        a, mid = mixer.conv_forward(x[:, :cut], w, None, True, None, mixer.rows(1, cut))
        c, last = mixer.conv_forward(x[:, cut:], w, None, True, mid, mixer.rows(1, 9 - cut))
        assert torch.equal(torch.cat([a, c], 1), whole) and torch.equal(last, end)


def test_packed_sequences_are_separate():
    x, w, init = randn(1, 10, 3, seed=1), randn(3, 4, seed=2), randn(4, 3, 3, seed=3)
    starts = [0, 1, 3, 7, 10]
    y, end = mixer.conv_forward(x, w, None, True, init, mixer.packed(starts))
    for k, (lo, hi) in enumerate(zip(starts, starts[1:])):
        a, f = mixer.conv_forward(x[:, lo:hi], w, None, True, init[k:k + 1], mixer.rows(1, hi - lo))
        assert torch.equal(a, y[:, lo:hi]) and torch.equal(f[0], end[k])
