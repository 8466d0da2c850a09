"""Rotary positions against complex products in float64.

An angle's fraction of a turn is rounded to float32 (its sine and cosine move by at most
pi 2^-24), sine and cosine are within 2 units of 2^-24, and the products and their sum add
2 more: 8 * 2^-24 (|a| + |b|) amplitude in all, and half a step of the output's type."""
import math

import pytest
import torch

from paper_2504_06949_amd import ops
from tests._helpers import ensure_built

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def turn(x, rope, pos, inverse=False):
    """(value, tolerance without the type's half step) in float64; pos [B or 1, L]."""
    rot, half = rope.rot, rope.rot // 2
    t = pos.double()[:, None, :, None] * rope.turns.double()
    ang = (t - t.round()) * (2 * math.pi) * (-1 if inverse else 1)
    x = x.double()
    out, tol = x.clone(), torch.zeros_like(x)
    a, b = (x[..., :half], x[..., half:rot]) if rope.layout == 0 else (x[..., 0:rot:2], x[..., 1:rot:2])
    z = torch.complex(a, b) * torch.polar(torch.full_like(ang, rope.amplitude), ang)
    lim = 8 * E * (a.abs() + b.abs()) * rope.amplitude
    if rope.layout == 0:
        out[..., :half], out[..., half:rot] = z.real, z.imag
        tol[..., :half], tol[..., half:rot] = lim, lim
    else:
        out[..., 0:rot:2], out[..., 1:rot:2] = z.real, z.imag
        tol[..., 0:rot:2], tol[..., 1:rot:2] = lim, lim
    return out, tol


def close(got, ref, rot):
    want, tol = ref
    err = (got.double() - want).abs()
    lim = tol + torch.finfo(got.dtype).eps / 2 * want.abs()
    assert (err <= lim + 1e-30).all(), f"worst {float((err / (lim + 1e-30)).max()):.2f} of the limit"
    assert torch.equal(got[..., rot:].double(), want[..., rot:])


def _x(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (128, 96), (64, 2), (64, 30), (80, 80), (2, 2),
                                   (66, 34), (256, 20)])
def test_head_sizes(d, rot, layout, dtype):
    print(f"case: rotary d={d} rot={rot} {layout} {dtype}", flush=True)
    rope = ops.Rotary(rot, layout=layout, amplitude=1.25)
    q, k = _x((2, 3, 37, d), dtype, 1), _x((2, 2, 37, d), dtype, 2)
    pos = torch.tensor([[0], [1000]], device="cuda") + torch.arange(37, device="cuda")
    a, b = rope.forward(q, k, positions=pos)
    close(a, turn(q, rope, pos), rot)
    close(b, turn(k, rope, pos), rot)
    a, b = rope.backward(q, k, positions=pos)
    close(a, turn(q, rope, pos, True), rot)
    close(b, turn(k, rope, pos, True), rot)


@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", {"factor": 4.0}), ("base", {"factor": 8.0}),
                                        ("ramp", {"factor": 32.0, "train_len": 4096})])
def test_scaled_frequencies_and_far_positions(scaling, kw):
    """Positions up to 2^31 - 1 and negative ones, int32 and int64, single and per sequence."""
    rope = ops.Rotary(64, scaling=scaling, **kw)
    assert rope.amplitude == (0.1 * math.log(32.0) + 1.0 if scaling == "ramp" else 1.0)
    pos = torch.tensor([0, 1, 63, 4096, 1000003, (1 << 31) - 1, -17, -(1 << 30)], device="cuda")
    q = _x((2, 4, 8, 64), torch.float32, 3)
    for p in (pos, pos.int(), torch.stack([pos, pos.flip(0)])):
        a, none = rope.forward(q, positions=p)
        assert none is None
        close(a, turn(q, rope, p if p.dim() == 2 else p[None]), 64)
    a, _ = rope.forward(q, start=1 << 30)
    close(a, turn(q, rope, (torch.arange(8, device="cuda") + (1 << 30))[None]), 64)


@pytest.mark.parametrize("B,H,Hk,L", [(1, 1, 1, 1), (16, 12, 12, 1), (1, 32, 4, 3), (2, 24, 24, 700), (1, 3, 1, 20001)])
def test_batches(B, H, Hk, L):
    print(f"case: rotary {B} {H} {Hk} {L}", flush=True)
    rope = ops.Rotary(64)
    q, k = _x((B, H, L, 64), torch.bfloat16, 4), _x((B, Hk, L, 64), torch.bfloat16, 5)
    a, b = rope.forward(q, k)
    pos = torch.arange(L, device="cuda")[None]
    close(a, turn(q, rope, pos), 64)
    close(b, turn(k, rope, pos), 64)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_strides_and_in_place(layout):
    rope = ops.Rotary(48, layout=layout)
    fused = _x((2, 50, 3, 4, 64), torch.bfloat16, 6)
    q, k = fused[:, :, 0].transpose(1, 2), fused[:, :, 1].transpose(1, 2)
    want = rope.forward(q.contiguous(), k.contiguous())
    got = rope.forward(q, k)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    rest = fused[:, :, 2].clone()
    rope.forward(q, k, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[:, :, 2], rest)
    # one of the two in place: the other still gets the features that are not turned
    q, k = _x((1, 2, 9, 64), torch.bfloat16, 7), _x((1, 2, 9, 64), torch.bfloat16, 8)
    want = rope.forward(q, k)
    other = torch.zeros_like(k)
    rope.forward(q, k, out=(q, other))
    assert torch.equal(q, want[0]) and torch.equal(other, want[1])


def test_odd_alignment_and_empty():
    rope = ops.Rotary(32)
    buf = _x((1, 2, 5, 67), torch.bfloat16, 9)
    x = buf[..., 3:]                                     # rows at odd element offsets
    close(rope.forward(x)[0], turn(x, rope, torch.arange(5, device="cuda")[None]), 32)
    q, k = rope.forward(torch.empty((1, 2, 0, 64), device="cuda"), torch.empty((1, 0, 0, 64), device="cuda"))
    assert q.shape == (1, 2, 0, 64) and k.shape == (1, 0, 0, 64)


def test_autograd():
    rope = ops.Rotary(64, layout="interleaved", scaling="ramp", factor=4.0, train_len=64)
    q = _x((2, 3, 20, 64), torch.float32, 1).requires_grad_(True)
    k = _x((2, 1, 20, 64), torch.float32, 2).requires_grad_(True)
    pos = torch.arange(20, device="cuda")
    a, b = rope(q, k.expand(2, 3, 20, 64), pos)          # a key head shared by broadcasting
    dq, dk = _x(a.shape, torch.float32, 3), _x(b.shape, torch.float32, 4)
    ((a * dq).sum() + (b * dk).sum()).backward()
    close(q.grad, turn(dq, rope, pos[None], True), 64)
    want, tol = turn(dk, rope, pos[None], True)
    assert ((k.grad.double() - want.sum(1, keepdim=True)).abs()
            <= tol.sum(1, keepdim=True) + 4 * E * want.abs().sum(1, keepdim=True)).all()
    one = _x((2, 3, 20, 64), torch.float32, 1).requires_grad_(True)
    rope(one)[0].sum().backward()
    close(one.grad, turn(torch.ones_like(one), rope, pos[None], True), 64)


def test_captured_step():
    """Turned in place and back in a graph, replayed with new contents between eager calls."""
    rope = ops.Rotary(64)
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((1, 4, 70, 64), generator=g, device="cuda").bfloat16()
    k = torch.randn((1, 2, 70, 64), generator=g, device="cuda").bfloat16()
    pos = torch.arange(70, device="cuda")

    def step():
        a, b = rope.forward(q, k, pos)
        return a, b, *rope.backward(a, b, pos)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        q.copy_(q.roll(1, 2))
        k.copy_(k.roll(1, 2))
        pos.add_(1000)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_second_derivatives_are_refused():
    rope = ops.Rotary(64)
    q = torch.ones((1, 1, 3, 64), device="cuda", requires_grad=True)
    g, = torch.autograd.grad((rope(q)[0] ** 2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
