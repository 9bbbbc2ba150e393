"""The layer of volume_block.py, all operators one behind the other: result and gradients against the same formulas in 64 bits, and against
differences; a step captured into a graph."""
import pytest
import torch

from paper_1606_05688_amd import volume_block
from paper_1606_05688_amd.volume_block import VolumeLayer

pytestmark = pytest.mark.gpu


def _turn(x, pos, freq, sections):
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    R = len(axis)
    t = (pos.double()[:, axis] * freq)[:, None]
    u, v = x[..., :R], x[..., R:2 * R]
    return torch.cat((u * t.cos() - v * t.sin(), u * t.sin() + v * t.cos(), x[..., 2 * R:]), -1)


def _plain(layer, w, x, pos, lens, left, right, sinks):
    n = lambda a: a / torch.sqrt((a * a).mean(-1, keepdim=True) + 1e-5)  # noqa: E731
    Hq, Hk, D = layer.Hq, layer.Hk, layer.D
    qkv = ((n(x) * w["pre1"]) @ w["wqkv"].T + w["bqkv"]).view(len(x), -1, D)
    q, k = (_turn(y, pos, layer.freq.double().cpu(), layer.sections) for y in (qkv[:, :Hq], qkv[:, Hq:Hq + Hk]))
    v, outs, at = qkv[:, Hq + Hk:], [], 0
    for m in lens:
        i = torch.arange(m)
        see = (i[None] <= i[:, None] + right) & ((i[None] >= i[:, None] - left) | (i[None] < sinks))
        s = torch.einsum("ihd,jhd->hij", q[at:at + m], k[at:at + m].repeat_interleave(Hq // Hk, 1)) * D ** -0.5
        outs.append(torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(~see, -torch.inf), -1), v[at:at + m].repeat_interleave(Hq // Hk, 1)))
        at += m
    h = x + w["gate"] * w["post"] * n(torch.cat(outs).reshape(len(x), -1) @ w["wo"].T)
    return h + torch.nn.functional.gelu((n(h) * w["pre2"]) @ w["w1"].T + w["b1"]) @ w["w2"].T + w["b2"]


def _case(dtype):
    layer, lens = VolumeLayer(Hq=6, Hk=2, D=16, sections=(3, 2, 2), dtype=dtype, seed=1), [70, 1, 0, 45]
    g = torch.Generator(device="cuda").manual_seed(2)
    T = sum(lens)
    x, dout = (torch.randn((T, 96), generator=g, device="cuda").to(dtype) for _ in range(2))
    pos = torch.randint(-20, 90, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    cu = torch.tensor([0, 70, 71, 71, 116], dtype=torch.int32, device="cuda")
    return layer, lens, x, dout, pos, cu, dict(left=20, right=1, sinks=3)


# Relative to a tensor's norm.  fp32: sums of up to 400 terms are off by 400 * 2^-24 of their terms' magnitudes, which are at most ten times a
# result here, through ten operators.  16-bit types: half a step for each result, and for what is rounded before a product, of the ten.
BOUND = {torch.float32: 10 * 10 * 400 * 2.0 ** -24, torch.bfloat16: 20 * 2.0 ** -8, torch.float16: 20 * 2.0 ** -11 + 10 * 10 * 400 * 2.0 ** -24}


@pytest.mark.parametrize("dtype", list(BOUND))
def test_result_and_gradients(dtype):
    layer, lens, x, dout, pos, cu, window = _case(dtype)
    out, kept = layer.forward(x, pos, cu, max(lens), **window)
    dx, grads = layer.backward(dout, kept)
    w = {k: t.double().cpu().requires_grad_() for k, t in layer.weights.items()}
    xr = x.double().cpu().requires_grad_()
    exp = _plain(layer, w, xr, pos.cpu(), lens, **window)
    exp.backward(dout.double().cpu())
    assert set(grads) == set(w)
    for name, a, b in [("out", out, exp.detach()), ("x", dx, xr.grad)] + [(k, grads[k], w[k].grad) for k in w]:
        assert a.dtype == dtype and a.shape == b.shape
        off = ((a.double().cpu() - b).norm() / b.norm()).item()
        assert off <= BOUND[dtype], f"{name}: {off:.3g}"


def test_differences():
    layer, lens, x, dout, pos, cu, window = _case(torch.float32)
    f = lambda y: (layer.forward(y, pos, cu, max(lens), **window)[0].double() * dout.double()).sum().item()  # noqa: E731
    dx, grads = layer.backward(dout, layer.forward(x, pos, cu, max(lens), **window)[1])
    way = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    for target, grad in ((x, dx), (layer.weights["wqkv"], grads["wqkv"]), (layer.weights["w1"], grads["w1"])):
        step = torch.randn(target.shape, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
        step *= target.norm() / step.norm()
        ends = []
        for s in (-1, 1):
            target += s * 2.0 ** -9 * step
            ends.append(f(x))
            target -= s * 2.0 ** -9 * step
        exp = (grad.double() * step.double()).sum().item()
        # second differences of a function whose size is |out| |dout|: the step squared times a third derivative of its size; its fp32 errors over the step
        size = (layer.forward(x, pos, cu, max(lens), **window)[0].double().norm() * dout.double().norm()).item()
        assert abs((ends[1] - ends[0]) * 2.0 ** 8 - exp) <= size * (100 * 2.0 ** -18 + 400 * 2.0 ** -24 * 2.0 ** 8)


def test_graph():
    layer, lens, x, dout, pos, cu, window = _case(torch.bfloat16)

    def step():
        out, kept = layer.forward(x, pos, cu, max(lens), **window)
        dx, grads = layer.backward(dout, kept)
        return [out, dx, *grads.values()]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held))


def test_command(capsys):
    volume_block.main()
    assert "gradients of size" in capsys.readouterr().out
