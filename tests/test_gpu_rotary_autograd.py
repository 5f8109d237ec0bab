"""rotary() within a graph of gradients, and what it refuses there."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_cache import BF, FP, gen, i32, normal   # noqa: E402

import paper_2410_03355_b200 as lt   # noqa: E402

pytestmark = pytest.mark.gpu


def made(dtype=FP, B=2, R=9, H=3, D=64, sections=(10, 12), interleaved=False, seed=400):
    x = normal((B, R, H, D), seed, dtype)
    pos = i32(torch.randint(0, 5000, (len(sections), B, R), generator=gen(seed + 1)))
    return x, pos, lt.Rotation((10000.0 ** (-torch.arange(sum(sections)) / sum(sections))).cuda(), sections, interleaved=interleaved)


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradient(interleaved, inverse, dtype):
    x, pos, rot = made(dtype, interleaved=interleaved)
    plain = lt.rotary(x, pos, rot, inverse=inverse)
    x.requires_grad_()
    y = lt.rotary(x, pos, rot, inverse=inverse)
    assert y.requires_grad and torch.equal(y, plain)
    g = normal(y.shape, 410, dtype)
    (grad,) = torch.autograd.grad(y, x, g)
    assert torch.equal(grad, lt.rotary(g, pos, rot, inverse=not inverse))
    # f(x) = sum(g * rotary(x)) is linear: differences of it are its gradient up to roundings (in fp32; each of the eight below of values under 8, 2^-24 of them)
    if dtype == FP:
        f = lambda z: (lt.rotary(z, pos, rot, inverse=inverse).double() * g.double()).sum()   # noqa: E731
        with torch.no_grad():
            for i in (0, 9, 10, 21, 22, 43, 44, 63, 1000):
                d = torch.zeros_like(x).view(-1)
                d[i] = 1.0
                assert abs((f(x + d.view_as(x)) - f(x - d.view_as(x))) / 2 - grad.view(-1)[i].double()) < 2 * 5 * 8 * (8 * 2.0 ** -24 + 2 * 2.0 ** -21)


def test_gradients_of_any_strides():
    """A sum's gradient is one number expanded; a transposed product's has strides of its own; rows of a fused projection get theirs in place."""
    x, pos, rot = made()
    x.requires_grad_()
    lt.rotary(x, pos, rot).sum().backward()
    want = lt.rotary(torch.ones_like(x), pos, rot, inverse=True)
    assert torch.equal(x.grad, want)
    g = normal((64, 3, 9, 2), 420).permute(3, 2, 1, 0)
    (grad,) = torch.autograd.grad(lt.rotary(x, pos, rot), x, g)
    assert torch.equal(grad, lt.rotary(g.contiguous(), pos, rot, inverse=True))
    fused = normal((2, 9, 7, 65), 421).requires_grad_()
    lt.rotary(fused[:, :, 2:5, 1:], pos, rot).sum().backward()
    assert torch.equal(fused.grad[:, :, 2:5, 1:], want) and not fused.grad[:, :, :2].any() and not fused.grad[..., 0].any()


def test_gradient_of_the_gradient():
    x, pos, rot = made()
    g = normal(x.shape, 430).requires_grad_()
    x.requires_grad_()
    (grad,) = torch.autograd.grad(lt.rotary(x, pos, rot), x, g, create_graph=True)
    w = normal(x.shape, 431)
    (back,) = torch.autograd.grad(grad, g, w)
    assert torch.equal(back, lt.rotary(w, pos, rot))


def test_as_part_of_a_step():
    """Weights in front of it are trained through it; a call on another stream belongs there, its gradient too."""
    x, pos, rot = made(D=64)
    w = normal((64, 64), 440, spread=0.1).requires_grad_()
    side = torch.cuda.Stream()
    lt.rotary(x @ w, pos, rot).square().sum().backward()
    want = w.grad.clone()
    y = lt.rotary(x, pos, rot)
    # |rotary(x w)|^2 = |x w|^2 in the formula.  In 32 bits: a product of 64, two turns (each 3 roundings and 2^-21 of the pair), a sum of 54; by magnitude
    exact = 2 * torch.einsum("brhi,brhj->ij", x.double(), x.double() @ w.detach().double())
    size = 4 * torch.einsum("brhi,brh->i", x.double().abs(), (x.double().abs() @ w.detach().double().abs()).amax(-1))[:, None]
    assert ((want.double() - exact).abs() <= size * (200 * 2.0 ** -24 + 2.0 ** -20)).all()
    del y
    w.grad = None
    side.wait_stream(torch.cuda.current_stream())
    out = lt.rotary(x @ w, pos, rot, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    out.square().sum().backward()
    torch.cuda.synchronize()
    assert torch.equal(w.grad, want)


def test_positions_that_change_before_the_gradient_are_noticed():
    x, pos, rot = made()
    x.requires_grad_()
    y = lt.rotary(x, pos, rot)
    pos.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_results_in_place_have_no_gradient():
    x, pos, rot = made()
    leaf = x.clone().requires_grad_()
    for out in (torch.empty_like(x), leaf):
        with pytest.raises(ValueError, match="gradient"):
            lt.rotary(leaf, pos, rot, out=out)
    with pytest.raises(ValueError, match="gradient"):
        lt.rotary(x, pos, rot, out=leaf)
    with torch.no_grad():
        assert torch.equal(lt.rotary(leaf, pos, rot, out=torch.empty_like(x)), lt.rotary(x, pos, rot))
    with torch.inference_mode():
        assert not lt.rotary(leaf, pos, rot).requires_grad


def test_gradient_recorded_and_replayed():
    x, pos, rot = made()
    g = normal(x.shape, 450)
    static = x.clone()

    def step():
        leaf = static.detach().requires_grad_()
        return torch.autograd.grad(lt.rotary(leaf, pos, rot), leaf, g)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grad = step()
    g.copy_(normal(x.shape, 451))
    pos.add_(3)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(grad, lt.rotary(g, pos, rot, inverse=True))


def test_inverse_is_a_truth_value():
    x, pos, rot = made()
    back = lt.rotary(x, pos, rot, inverse=True)
    strided = torch.zeros((2, 9, 3, 65), device="cuda")[..., 1:]
    for yes in (1, 0.5, "x"):
        assert torch.equal(lt.rotary(x, pos, rot, inverse=yes), back)
        assert torch.equal(lt.rotary(x, pos, rot, inverse=yes, out=strided), back)
        assert torch.equal(lt.rotary(x, pos, rot, inverse=yes, stream=torch.cuda.current_stream()), back)
    for unclear in (torch.zeros(2), torch.zeros(2, device="cuda")):
        with pytest.raises(RuntimeError, match="ambiguous"):
            lt.rotary(x, pos, rot, inverse=unclear)
