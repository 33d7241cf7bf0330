"""Plain float64 definitions (torch, CPU) of what stands around the layer in a
block: the short convolution, the selective scan and the residual addition with
norm, with their gradients.

Token by token and sequence by sequence; ``spans`` lists the sequences as (row,
first token, end).  A tensor may be of any type; everything is widened first.
"""
from __future__ import annotations

import torch


def _f64(t):
    return None if t is None else t.detach().cpu().double()


def rows(b, T):
    """The sequences of a batch of plain rows."""
    return [(r, 0, T) for r in range(b)]


def packed(starts):
    """The sequences of one packed row."""
    return [(0, lo, hi) for lo, hi in zip(starts, starts[1:])]


def _silu(v):
    return v * torch.sigmoid(v)


def _silu_grad(v):
    s = torch.sigmoid(v)
    return s * (1 + v * (1 - s))


def conv_forward(x, weight, bias, silu, init, spans):
    """(y, final states)."""
    x, w, bias, init = _f64(x), _f64(weight), _f64(bias), _f64(init)
    C, W = w.shape
    y, final = torch.zeros_like(x), x.new_zeros(len(spans), W - 1, C)
    for k, (r, lo, hi) in enumerate(spans):
        before = init[k] if init is not None else x.new_zeros(W - 1, C)
        line = torch.cat([before, x[r, lo:hi]])
        v = sum(line[j:j + hi - lo] * w[:, j] for j in range(W)) + (bias if bias is not None else 0.0)
        y[r, lo:hi] = _silu(v) if silu else v
        final[k] = line[hi - lo:]
    return y, final


def conv_backward(x, weight, bias, silu, init, spans, dy, dfinal):
    x, w, bias, init, dy, dfinal = (_f64(t) for t in (x, weight, bias, init, dy, dfinal))
    C, W = w.shape
    g = {"dx": torch.zeros_like(x), "dweight": torch.zeros_like(w), "dbias": w.new_zeros(C),
         "dinit": x.new_zeros(len(spans), W - 1, C)}
    for k, (r, lo, hi) in enumerate(spans):
        before = init[k] if init is not None else x.new_zeros(W - 1, C)
        line = torch.cat([before, x[r, lo:hi]])
        v = sum(line[j:j + hi - lo] * w[:, j] for j in range(W)) + (bias if bias is not None else 0.0)
        dv = dy[r, lo:hi] * (_silu_grad(v) if silu else 1.0)
        dline = torch.zeros_like(line)
        for j in range(W):
            dline[j:j + hi - lo] += dv * w[:, j]
            g["dweight"][:, j] += (dv * line[j:j + hi - lo]).sum(0)
        g["dbias"] += dv.sum(0)
        if dfinal is not None:
            dline[hi - lo:] += dfinal[k]
        g["dinit"][k], g["dx"][r, lo:hi] = dline[:W - 1], dline[W - 1:]
    return g


def _scan_inputs(x, dt, A_log, B, C, D, dt_bias, softplus):
    x, dt, A_log, B, C, D, dt_bias = (_f64(t) for t in (x, dt, A_log, B, C, D, dt_bias))
    E = x.shape[-1]
    v = dt + (dt_bias if dt_bias is not None else 0.0)
    d = torch.logaddexp(v, torch.zeros_like(v)) if softplus else v
    of = torch.arange(E) // (E // B.shape[-2])     # the group of every channel
    return x, v, d, -torch.exp(A_log), B, C, D if D is not None else x.new_zeros(E), of


def scan_forward(x, dt, A_log, B, C, D, z, dt_bias, softplus, init, spans):
    """(y, final states)."""
    x, v, d, A, B, C, D, of = _scan_inputs(x, dt, A_log, B, C, D, dt_bias, softplus)
    z, init = _f64(z), _f64(init)
    y, final = torch.zeros_like(x), x.new_zeros(len(spans), *A.shape)
    for k, (r, lo, hi) in enumerate(spans):
        h = init[k] if init is not None else torch.zeros_like(A)
        for t in range(lo, hi):
            h = torch.exp(d[r, t, :, None] * A) * h + (d[r, t] * x[r, t])[:, None] * B[r, t, of]
            y[r, t] = (h * C[r, t, of]).sum(-1) + D * x[r, t]
        final[k] = h
    return (y * _silu(z) if z is not None else y), final


def scan_backward(x, dt, A_log, B, C, D, z, dt_bias, softplus, init, spans, dy, dfinal):
    x, v, d, A, B, C, D, of = _scan_inputs(x, dt, A_log, B, C, D, dt_bias, softplus)
    z, init, dy, dfinal = (_f64(t) for t in (z, init, dy, dfinal))
    G, N = B.shape[-2:]
    E = x.shape[-1]
    g = {"dx": torch.zeros_like(x), "ddt": torch.zeros_like(x), "dB": torch.zeros_like(B), "dC": torch.zeros_like(C),
         "dz": torch.zeros_like(x), "dA_log": torch.zeros_like(A), "dD": x.new_zeros(E), "ddt_bias": x.new_zeros(E),
         "dinit": x.new_zeros(len(spans), E, N)}
    for k, (r, lo, hi) in enumerate(spans):
        states = [init[k] if init is not None else torch.zeros_like(A)]
        for t in range(lo, hi):
            states.append(torch.exp(d[r, t, :, None] * A) * states[-1] + (d[r, t] * x[r, t])[:, None] * B[r, t, of])
        later = dfinal[k] if dfinal is not None else torch.zeros_like(A)
        for t in range(hi - 1, lo - 1, -1):
            h, before, a = states[t - lo + 1], states[t - lo], torch.exp(d[r, t, :, None] * A)
            dout = dy[r, t]
            if z is not None:
                g["dz"][r, t] = dout * ((h * C[r, t, of]).sum(-1) + D * x[r, t]) * _silu_grad(z[r, t])
                dout = dout * _silu(z[r, t])
            dh = later + dout[:, None] * C[r, t, of]
            g["dC"][r, t] = (dout[:, None] * h).view(G, E // G, N).sum(1)
            g["dB"][r, t] = (dh * (d[r, t] * x[r, t])[:, None]).view(G, E // G, N).sum(1)
            du, q = (dh * B[r, t, of]).sum(-1), dh * a * before
            g["dx"][r, t] = du * d[r, t] + D * dout
            g["dD"] += dout * x[r, t]
            dd = du * x[r, t] + (q * A).sum(-1)
            g["ddt"][r, t] = dd * torch.sigmoid(v[r, t]) if softplus else dd
            g["dA_log"] += q * d[r, t, :, None] * A
            later = dh * a
        g["dinit"][k] = later
    g["ddt_bias"] = g["ddt"].sum((0, 1))
    return g


def add_norm(x, weight, residual, eps):
    """(y, r)."""
    x, w, residual = _f64(x), _f64(weight), _f64(residual)
    r = x + residual if residual is not None else x
    y = r / torch.sqrt(r.square().mean(-1, keepdim=True) + eps)
    return (y * w if w is not None else y), r


def add_norm_backward(dy, r, weight, dresidual, eps):
    dy, r, w, dresidual = (_f64(t) for t in (dy, r, weight, dresidual))
    C = r.shape[-1]
    rstd = 1 / torch.sqrt(r.square().mean(-1, keepdim=True) + eps)
    n, g = r * rstd, dy * w if w is not None else dy
    d = rstd * (g - n * (g * n).mean(-1, keepdim=True))
    if dresidual is not None:
        d = d + dresidual
    return {"dx": d, "dresidual": d, "dweight": (dy * n).reshape(-1, C).sum(0)}
