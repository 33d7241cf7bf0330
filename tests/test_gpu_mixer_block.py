"""The operators around the layer together, as a block uses them: norm, projection
(a plain product here), convolution, scan or SSD layer; prompts continued token by
token, and gradients through the chain."""
import pytest
import torch

from oracle import mixer
from tests.mixer_harness import TOL, Draw, announce, check, off, seq_idx_of, ssd
from tests.test_gpu_parity import _gpu  # noqa: F401

pytestmark = pytest.mark.gpu

H, P, N, G, W, DM = 4, 64, 64, 1, 4, 96       # the layer's heads; model width
E = H * P


def params(seed=11):
    n = Draw(seed)
    conv = E + 2 * G * N
    return {"norm": 1 + n(DM, scale=0.1), "in": n(DM, E + conv + H, scale=DM ** -0.5), "conv_w": n(conv, W, scale=0.5),
            "conv_b": n(conv, scale=0.1), "A_log": n(H).abs(), "D": n(H), "dt_bias": n(H) - 2,
            "gate_norm": 1 + n(E, scale=0.1), "out": n(E, DM, scale=E ** -0.5)}


def ssd_block(w, x, res, conv_state=None, ssm_state=None, step=False):
    """norm -> projection -> convolution -> SSD layer with its gate and norm -> projection."""
    y, res = ssd.add_norm(x, w["norm"], residual=res)
    p = y.float() @ w["in"]                      # z, convolution's channels, dt
    z, xbc, dt = p[..., :E], p[..., E:E + E + 2 * G * N], p[..., -H:].contiguous()
    layer = dict(D=w["D"], dt_bias=w["dt_bias"], norm_weight=w["gate_norm"], norm_group_size=E)
    if step:     # the layer's token: one decode step, gate and norm as the definitions have them
        xbc = ssd.conv_step(xbc, w["conv_w"], conv_state, bias=w["conv_b"])
        xs, B, C = (t.contiguous() for t in torch.split(xbc, (E, G * N, G * N), -1))
        b = x.shape[0]
        d = torch.nn.functional.softplus(dt + w["dt_bias"])
        y = ssd.decode_step(xs.view(b, H, P), d, w["A_log"], B.view(b, G, N), C.view(b, G, N), ssm_state, D=w["D"])
        y = y.reshape(b, E) * torch.nn.functional.silu(z)
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5) * w["gate_norm"]
        return y @ w["out"], res, conv_state, ssm_state
    b, T = x.shape[:2]
    (xs, B, C), conv_state = ssd.conv_forward(xbc, w["conv_w"], bias=w["conv_b"], initial_states=conv_state,
                                              split=(E, G * N, G * N))
    y, ssm_state = ssd.forward_block(xs.view(b, T, H, P), dt, w["A_log"], B.view(b, T, G, N), C.view(b, T, G, N),
                                     z=z.contiguous().view(b, T, H, P), initial_states=ssm_state, **layer)
    return y.reshape(b, T, E) @ w["out"], res, conv_state, ssm_state


def test_ssd_block_prompt_then_tokens():
    announce("block with the SSD layer: prompt, then tokens")
    w, n = params(), Draw(12)
    x, res = n(2, 40, DM), n(2, 40, DM)
    whole = ssd_block(w, x, res)
    head = ssd_block(w, x[:, :33].contiguous(), res[:, :33].contiguous())
    states, out = head[2:], [head[0]]
    for t in range(33, 40):
        y, _, *states = ssd_block(w, x[:, t].contiguous(), res[:, t].contiguous(), *states, step=True)
        out.append(y[:, None])
    # float32 throughout: the layer's own tolerance (1e-4), for both sides
    assert off(torch.cat(out, 1), whole[0].cpu()) <= 2e-4
    for a, b in zip(states, whole[2:]):
        assert off(a, b.cpu()) <= 2e-4


def scan_block(w, x, res, conv_state=None, state=None, step=False):
    """norm (8-bit output and scales) -> projection -> convolution -> selective scan."""
    q, scale, res = ssd.add_norm_q8(x, w["norm"], residual=res, dtype=torch.int8)
    p = (q.float() @ w["in"][:, :2 * E]) * scale[..., None]
    xs, z = p[..., :E], p[..., E:]
    if step:
        xs = ssd.conv_step(xs, w["conv_w"][:E], conv_state, bias=w["conv_b"][:E])
    else:
        xs, conv_state = ssd.conv_forward(xs, w["conv_w"][:E].contiguous(), bias=w["conv_b"][:E],
                                          initial_states=conv_state)
    low = xs @ w["x"]                            # dt's low rank part, B, C: slices
    dt, B, C = low[..., :8] @ w["dt"], low[..., 8:24].unsqueeze(-2), low[..., 24:40].unsqueeze(-2)
    args = dict(D=w["skip"], z=z, dt_bias=w["scan_bias"])
    if step:
        y = ssd.scan_step(xs, dt, w["scan_A"], B, C, state, **args)
    else:
        y, state = ssd.scan_forward(xs, dt, w["scan_A"], B, C, initial_states=state, **args)
    return y @ w["out"], res, conv_state, state


def scan_params():
    w, n = params(), Draw(13)
    w["in"] = n(DM, 2 * E, scale=DM ** -0.5)
    w.update(x=n(E, 40, scale=E ** -0.5), dt=n(8, E, scale=0.3), skip=n(E), scan_bias=n(E) - 3,
             scan_A=torch.log(torch.arange(1, 17).float()).cuda().repeat(E, 1), conv_w=n(E, W, scale=0.5))
    return w


def test_scan_block_prompt_then_tokens():
    announce("block with the selective scan and an 8-bit norm: prompt, then tokens")
    w, n = scan_params(), Draw(14)
    x, res = n(2, 150, DM), n(2, 150, DM)
    whole = scan_block(w, x, res)
    head = scan_block(w, x[:, :140].contiguous(), res[:, :140].contiguous())
    states, out = head[2:], [head[0]]
    for t in range(140, 150):
        y, _, *states = scan_block(w, x[:, t].contiguous(), res[:, t].contiguous(), *states, step=True)
        out.append(y[:, None])
    assert off(torch.cat(out, 1), whole[0].cpu()) <= 2 * TOL[torch.float32]
    for a, b in zip(states, whole[2:]):
        assert off(a, b.cpu()) <= 2 * TOL[torch.float32]


@pytest.mark.parametrize("starts", [None, [0, 3, 90, 91, 170]])
def test_gradients_through_the_chain(starts):
    """norm -> convolution -> scan: each operator's gradient handed to the one before
    it, against the same chain of the definitions."""
    announce("gradients through norm, convolution and scan (%s)" % starts)
    n, T, C, S = Draw(15), 170, 24, 16
    x, res, wn = n(1, T, C), n(1, T, C), 1 + n(C, scale=0.1)
    wc, bc, A_log, D, bias = n(C, W, scale=0.5), n(C, scale=0.1), n(C, S), n(C), n(C) - 2
    dt, B, Cm, z, dy, dr = n(1, T, C), n(1, T, 1, S), n(1, T, 1, S), n(1, T, C), n(1, T, C), n(1, T, C)
    spans = mixer.packed(starts) if starts else mixer.rows(1, T)
    packed = {"seq_idx": seq_idx_of(starts), "nseq": len(spans)} if starts else {}
    y0, r = ssd.add_norm(x, wn, residual=res)
    y1, _ = ssd.conv_forward(y0, wc, bias=bc, **packed)
    scan = dict(D=D, z=z, dt_bias=bias)
    g2 = ssd.scan_backward(y1, dt, A_log, B, Cm, dy, **scan, **packed)
    g1 = ssd.conv_backward(y0, wc, g2["dx"], bias=bc, **packed)
    g0 = ssd.add_norm_backward(g1["dx"], r, wn, dresidual=dr)
    m0, mr = mixer.add_norm(x, wn, res, 1e-5)
    m1, _ = mixer.conv_forward(m0, wc, bc, True, None, spans)
    w2 = mixer.scan_backward(m1, dt, A_log, B, Cm, D, z, bias, True, None, spans, dy, None)
    w1 = mixer.conv_backward(m0, wc, bc, True, None, spans, w2["dx"], None)
    w0 = mixer.add_norm_backward(w1["dx"], mr, wn, dr, 1e-5)
    for got, want, names in ((g2, w2, ("dx", "ddt", "dz", "dB", "dC", "dA_log", "dD", "ddt_bias")),
                             (g1, w1, ("dx", "dweight", "dbias")), (g0, w0, ("dx", "dweight"))):
        for k in names:
            check(k, got[k], want[k], 3 * TOL[torch.float32])    # three operators' roundings


def test_two_calls_on_two_streams():
    """Two scans and two convolutions at once, with workspaces of their own."""
    announce("two calls at once")
    n = Draw(16)
    sets = [(n(2, 700, 130), n(2, 700, 130), n(130, 16), n(2, 700, 1, 16), n(2, 700, 1, 16)) for _ in range(2)]
    dys, wc = [n(2, 700, 130) for _ in range(2)], n(130, 4)
    alone = [(ssd.scan_forward(*s)[0], ssd.scan_backward(*s, d)["dA_log"], ssd.conv_backward(s[0], wc, d)["dweight"])
             for s, d in zip(sets, dys)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                s, d = sets[k], dys[k]
                got[k] = (ssd.scan_forward(*s)[0], ssd.scan_backward(*s, d)["dA_log"],
                          ssd.conv_backward(s[0], wc, d)["dweight"])
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
