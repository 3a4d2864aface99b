"""pa_dropout on the GPU against 64 bits and the published generator (ask_ref.py)."""
import numpy as np
import pytest
import torch

import ask_ref as R
from paper_2502_02414_amd import ops
from pa_cases import say

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DT = {"f32": F32, "bf16": BF16}


def expected(y, r, p, seed, offset):
    keep, scale = R.kept(np.arange(y.numel()), p, seed, offset)
    out = torch.where(keep, y.double().view(-1) * scale, 0.0)
    mag = out.abs()
    if r is not None:
        out, mag = out + r.double().view(-1), mag + r.double().view(-1).abs()
    # half a step of the type; the scale's, the product's and the sum's in 32 bits
    return out, R.half_step(y.dtype) * out.abs() * (1 + 2 ** -8) + 4 * R.U * mag + 1e-37, keep


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("resid", [False, True])
@pytest.mark.parametrize("n,p,seed,offset", [
    (1, 0.5, 0, 0), (7, 0.3, 1, 2), (8, 0.1, 5, 1), (9, 0.25, 2 ** 63 + 11, 2 ** 40 + 3),
    (256, 0.1, 3, 4), (2047, 0.9, 2 ** 64 - 1, 2 ** 64 - 1), (4096, 0.0, 9, 9),
    (100003, 0.05, 12345, 6), (70001, 65535 / 65536, 4, 4), (5000000, 0.5, 77, 1)])
def test_dropout(dt, resid, n, p, seed, offset):
    say(f"dropout {dt} n={n} p={p} resid={resid}")
    g = torch.Generator()
    g.manual_seed(n)
    y = torch.randn(n, generator=g).to(DT[dt])
    r = torch.randn(n, generator=g).to(DT[dt]) if resid else None
    out = torch.full((n,), 7.0, dtype=DT[dt], device="cuda")
    gy, gr = y.cuda(), None if r is None else r.cuda()
    ops.pa_dropout(gy, out, p, seed, offset, r=gr)
    ref, bound, keep = expected(y, r, p, seed, offset)
    assert ((out.cpu().double() - ref).abs() <= bound).all()
    # in place of either input: the same
    for at in ([gy, gr] if resid else [gy]):
        a, b = gy.clone(), None if gr is None else gr.clone()
        to = a if at is gy else b
        ops.pa_dropout(a, to, p, seed, offset, r=b)
        assert torch.equal(to, out)
    if n >= 100000 and 0.01 < p < 0.99:  # (five standard deviations)
        share = keep.double().mean().item()
        assert abs(share - (1 - p)) <= 5 * (p * (1 - p) / n) ** 0.5 + 2 ** -17


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_dropped_elements_are_not_read_into_the_result(dt):
    n = 3001
    y = torch.ones(n, dtype=DT[dt])
    keep, _ = R.kept(np.arange(n), 0.4, 3, 3)
    y[~keep] = torch.tensor([float("nan"), float("inf"), -float("inf")])[
        torch.arange(int((~keep).sum())) % 3].to(DT[dt])
    out = torch.empty(n, dtype=DT[dt], device="cuda")
    ops.pa_dropout(y.cuda(), out, 0.4, 3, 3)
    assert torch.isfinite(out).all() and (out.cpu()[~keep] == 0).all()
    bad = torch.full((n,), float("nan"), dtype=DT[dt], device="cuda")
    ops.pa_dropout(bad, out, 0.4, 3, 3)
    assert torch.equal(torch.isnan(out.cpu()), keep)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_backward_draws_the_same_numbers(dt):
    """The gradient of sum(w out), against differences of the forward (which is linear in
    y: whole steps of 1 and sizes that the type holds exactly)."""
    n = 10007
    y = torch.zeros(n, dtype=DT[dt], device="cuda")
    w = torch.randint(-8, 9, (n,), device="cuda").to(DT[dt])
    one, zero, dy = torch.empty_like(y), torch.empty_like(y), torch.empty_like(y)
    r = torch.zeros_like(y)
    ops.pa_dropout(y + 1, one, 0.5, 11, 7, r=r)
    ops.pa_dropout(y, zero, 0.5, 11, 7, r=r)
    ops.pa_dropout(w, dy, 0.5, 11, 7)
    assert torch.equal(dy, w * (one - zero))
    assert (dy != 0).float().mean() > 0.4


def test_elements_beyond_32_bits():
    """More than 2^31 elements: the ends against the definition."""
    n = (1 << 31) + 5 * 256 + 3
    y = torch.ones(n, dtype=BF16, device="cuda")
    out = torch.empty_like(y)
    ops.pa_dropout(y, out, 0.5, 1, 2)
    for at in (0, (1 << 31) - 1000, n - 1003):
        e = np.arange(at, at + 1003 if at + 1003 < n else n)
        keep, scale = R.kept(e, 0.5, 1, 2)
        assert torch.equal(out[at:at + len(e)].cpu().double(), keep.double() * scale)


def test_in_a_graph_with_the_offset_on_the_device():
    """Replays whose offset moves on: each the eager call's numbers, all different."""
    y = torch.randn(5000, device="cuda")
    r = torch.randn(5000, device="cuda")
    out, at = torch.empty_like(y), torch.zeros(1, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ops.pa_dropout(y, out, 0.3, 5, 100, r=r, offset_dev=at)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at.add_(1)
        ops.pa_dropout(y, out, 0.3, 5, 100, r=r, offset_dev=at)
    seen = []
    for rep in range(1, 6):
        eager = torch.empty_like(y)
        ops.pa_dropout(y, eager, 0.3, 5, 100 + rep, r=r)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), rep
        assert not any(torch.equal(out, b) for b in seen)
        seen.append(out.clone())


def test_on_another_stream():
    y = torch.randn(100000, device="cuda")
    a, b = torch.empty_like(y), torch.empty_like(y)
    ops.pa_dropout(y, a, 0.1, 1, 1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ops.pa_dropout(y, b, 0.1, 1, 1, stream=s)
    s.synchronize()
    assert torch.equal(a, b)
