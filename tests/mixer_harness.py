"""Helpers shared by the GPU tests of the convolution, the selective scan and the
norm.

``TOL``: what a result may be off, relative to the largest value of its tensor.
float32: chains and sums of up to 2,048 roundings of 2^-24 each, of terms no
larger than that value.  bfloat16: that, and the rounding of the result, half a
step (2^-8); operands are not rounded inside the kernels.
"""
import torch

from paper_2405_21060_amd import ssd  # noqa: F401
from tests.ssd_harness import announce  # noqa: F401

TOL = {torch.float32: 2048 * 2.0 ** -24, torch.bfloat16: 2048 * 2.0 ** -24 + 2.0 ** -8}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Draw:
    """Seeded normal tensors, drawn in float32 on the CPU and then cast."""

    def __init__(self, seed):
        self.gen = torch.Generator().manual_seed(seed)

    def __call__(self, *shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.gen) * scale).to(dtype).cuda()


def off(got, want):
    """max |got - want| / max |want|."""
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, (got.shape, want.shape)
    if not want.numel():
        return 0.0
    top = want.abs().max()
    return float((got - want).abs().max() / (top if top > 0 else 1.0))


def check(name, got, want, tol=None):
    e = off(got, want)
    tol = TOL[got.dtype] if tol is None else tol
    assert e <= tol, "%s: off by %.3e, %.3e allowed" % (name, e, tol)


def seq_idx_of(starts):
    n = torch.tensor([hi - lo for lo, hi in zip(starts, starts[1:])])
    return torch.repeat_interleave(torch.arange(len(n)), n).to(torch.int32).view(1, -1).cuda()


def same(a, b):
    """Bit for bit, through tuples and dicts."""
    if isinstance(a, dict):
        return all(same(a[k], b[k]) for k in a)
    if isinstance(a, (tuple, list)):
        return all(same(x, y) for x, y in zip(a, b))
    return a is None and b is None or torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def streams_and_graphs(call, reset=lambda: None):
    """``call`` eager, on a side stream, and captured and replayed three times with
    eager work in between: the same bits every time."""
    reset()
    first = call()
    first = _copy(first)
    side = torch.cuda.Stream()
    reset()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call()
    side.synchronize()
    assert same(first, second)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert same(first, held)
        reset()
        assert same(first, call())


def _copy(v):
    if isinstance(v, dict):
        return {k: _copy(x) for k, x in v.items()}
    if isinstance(v, (tuple, list)):
        return tuple(_copy(x) for x in v)
    return None if v is None else v.clone()
