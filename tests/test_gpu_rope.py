"""Rotary positions against complex multiplication in 64 bits: layouts, parts of the head, scalings, far and negative positions, views,
in place, and the transposed operator against the formula's gradient and against differences."""
import math

import pytest
import torch

import paper_2505_21136_amd as sage
from paged_ref import EPS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _freqs(plan):
    return torch.tensor([plan.turns[i] / 2.0 ** 64 for i in range(plan.rot // 2)], dtype=torch.float64), plan.magnitude


def _want(x, pos, plan, transposed=False):
    """(result, bound): the hardware's sine and cosine of an angle in turns are taken to be 2^-18 off at most (their argument is, after its own
    rounding, 2^-24), products and sums add 3 roundings of 2^-24: (|a| + |b|) magnitude (2^-18 + 2^-22)."""
    f, mag = _freqs(plan)
    x = x.double().cpu()
    n = plan.rot // 2
    i = torch.arange(n)
    a, b = (i, i + n) if plan.layout == 0 else (2 * i, 2 * i + 1)
    # position * turns modulo one, in whole numbers
    turns = torch.tensor([[((int(p) * plan.turns[k]) % 2 ** 64) / 2.0 ** 64 for k in range(n)] for p in pos.tolist()], dtype=torch.float64)
    z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.full_like(turns, mag), (-1 if transposed else 1) * 2 * math.pi * turns)[:, None]
    y, e = x.clone(), torch.zeros_like(x)
    y[..., a], y[..., b] = z.real, z.imag
    e[..., a] = e[..., b] = (x[..., a].abs() + x[..., b].abs()) * mag * (2.0 ** -18 + 2.0 ** -22)
    return y, e


def _check(got, want, err, dtype, what):
    tol = err + EPS[dtype] * (want.abs() + err) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert torch.isfinite(got.float()).all(), what
    worst = ((got.double().cpu() - want).abs() / tol.clamp(min=1e-300)).max().item()
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,far", [(1, 1, 0, 64, 64, 10), (1, 4, 1, 128, 128, 1 << 30), (7, 3, 2, 64, 16, 5000), (65, 5, 5, 128, 48, 1 << 22),
                                               (300, 32, 8, 128, 112, 1 << 17), (129, 1, 1, 64, 48, 1 << 31)])
def test_rotation(dtype, layout, T, Hq, Hkv, d, rot, far):
    g = torch.Generator().manual_seed(T + rot)
    plan = sage.rope_plan(rot, layout=layout, base=500000.0)
    pos = torch.randint(-far, far, (T,), generator=g).to(torch.int32)
    qkv = torch.randn(T, Hq + 2 * Hkv + 1, d, generator=g).to(dtype).to(DEV)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv] if Hkv else None        # views of a packed projection
    for transposed in (False, True):
        got = sage.sage_rope(q, pos.to(DEV), plan, k=k, transposed=transposed)
        for y, x, name in zip(got if Hkv else (got,), (q, k), "qk"):
            _check(y, *_want(x, pos, plan, transposed), dtype, f"{name} {transposed}")
    # in place, the same bits; the other heads of the projection stay
    before = qkv.clone()
    want = sage.sage_rope(q, pos.to(DEV), plan, k=k)
    sage.sage_rope(q, pos.to(DEV), plan, k=k, out=q, k_out=k)
    want = torch.cat(want, 1) if Hkv else want
    assert torch.equal(qkv[:, :Hq + Hkv].view(torch.int16), want.view(torch.int16))
    assert torch.equal(qkv[:, Hq + Hkv:].view(torch.int16), before[:, Hq + Hkv:].view(torch.int16))


@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("ntk", 8.0), ("yarn", 16.0), ("bands", 8.0), ("linear", 0.01)])
def test_scalings_and_many_tokens(scaling, factor):
    # enough rows that a wavefront takes several heads of a token, with heads that do not fill it
    T, Hq, Hkv, d = 9001, 13, 3, 64
    plan = sage.rope_plan(64, scaling=scaling, factor=factor, trained_len=2048)
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn(T, Hq, d, generator=g).to(torch.bfloat16).to(DEV), torch.randn(T, Hkv, d, generator=g).to(torch.bfloat16).to(DEV)
    pos = torch.arange(T, dtype=torch.int32) * 37
    qo, ko = sage.sage_rope(q, pos.to(DEV), plan, k=k)
    pick = torch.randperm(T, generator=g)[:200]
    _check(qo[pick.to(DEV)], *_want(q[pick.to(DEV)], pos[pick], plan), torch.bfloat16, "q")
    _check(ko[pick.to(DEV)], *_want(k[pick.to(DEV)], pos[pick], plan), torch.bfloat16, "k")


def test_output_views_and_head_major_tensors():
    T, H, d = 33, 4, 128
    plan = sage.rope_plan(d)
    q = torch.randn(H, T, d, device=DEV).half().transpose(0, 1)      # head-major
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    room = torch.full((T, H + 2, d), 7.0, dtype=torch.float16, device=DEV)
    out = sage.sage_rope(q, pos, plan, out=room[:, 1:H + 1])
    want = sage.sage_rope(q.contiguous(), pos, plan)
    assert torch.equal(out, want) and bool((room[:, 0] == 7).all()) and bool((room[:, H + 1] == 7).all())
    one = sage.sage_rope(q[:, :1].expand(T, H, d), pos, plan)          # a broadcast head
    assert torch.equal(one, want[:, :1].expand(T, H, d))


def test_transposed_is_the_gradient():
    T, H, d = 5, 2, 64
    g = torch.Generator().manual_seed(1)
    plan = sage.rope_plan(48, scaling="yarn", factor=4.0, trained_len=128, layout="interleaved")
    pos = torch.randint(0, 4000, (T,), generator=g).to(torch.int32)
    x, dy = torch.randn(T, H, d, generator=g).half(), torch.randn(T, H, d, generator=g).half()
    got = sage.sage_rope(dy.to(DEV), pos.to(DEV), plan, transposed=True)
    # the formula's gradient through autograd in 64 bits
    leaf = x.double().requires_grad_(True)
    f, mag = _freqs(plan)
    angle = 2 * math.pi * pos.double()[:, None] * f
    a, b = leaf[..., 0:48:2], leaf[..., 1:48:2]
    c, s = (mag * angle.cos())[:, None], (mag * angle.sin())[:, None]
    y = torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), leaf[..., 48:]], -1)
    y.backward(dy.double())
    _check(got, leaf.grad, _want(dy, pos, plan, True)[1] + 1e-9, torch.float16, "gradient")
    # and the kernel's own forward: <dy, F x> = <F^T dy, x>.  It is linear; both sides round to fp16: half a step an element at most
    fx = sage.sage_rope(x.to(DEV), pos.to(DEV), plan).double().cpu()
    lhs, rhs = (dy.double() * fx).sum(), (got.double().cpu() * x.double()).sum()
    slack = 2.0 ** -10 * ((dy.double() * fx).abs().sum() + (got.double().cpu() * x.double()).abs().sum())
    assert abs(lhs - rhs) <= slack
    # differences of the forward along a direction: linear, so any step is right; steps of 1 keep the rounding small beside it
    for i in (0, 1, 47, 50):
        e = torch.zeros_like(x)
        e[:, :, i] = 1.0
        diff = (sage.sage_rope((x + e).to(DEV), pos.to(DEV), plan).double().cpu() - sage.sage_rope((x).to(DEV), pos.to(DEV), plan).double().cpu())
        num = (diff * dy.double()).sum(-1)
        # two fp16 roundings of the forward's values (at most 8 here), one of x + e (at most 8), each 2^-11 relative
        room = 3 * 8 * 2.0 ** -11 * dy.double().abs().sum(-1) + 2.0 ** -10
        assert bool(((num - got.double().cpu()[..., i]).abs() <= room).all()), i


def test_other_stream_and_graph():
    T, H, d = 40, 6, 128
    plan = sage.rope_plan(64)
    q, pos = torch.randn(T, H, d, device=DEV).bfloat16(), torch.arange(T, dtype=torch.int32, device=DEV)
    want = sage.sage_rope(q, pos, plan)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sage.sage_rope(q, pos, plan)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out, graph = torch.zeros_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sage.sage_rope(q, pos, plan, out=out)
    for i in range(3):
        q.copy_(torch.randn(T, H, d, device=DEV).bfloat16())
        pos.add_(11)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, sage.sage_rope(q, pos, plan)), i


def test_refusals_on_the_device():
    q, pos, plan = torch.zeros(4, 2, 64, dtype=torch.float16, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), sage.rope_plan(64)
    for call in (lambda: sage.sage_rope(q, pos.long(), plan), lambda: sage.sage_rope(q, pos[:3], plan), lambda: sage.sage_rope(q.float(), pos, plan),
                 lambda: sage.sage_rope(q, pos, plan, k=q[:3]), lambda: sage.sage_rope(q[..., ::2], pos, plan), lambda: sage.sage_rope(q[0], pos, plan),
                 lambda: sage.sage_rope(q, pos, sage.rope_plan(128)), lambda: sage.sage_rope(q, pos, plan, out=q.float()),
                 lambda: sage.sage_rope(q, pos, plan, k_out=q), lambda: sage.sage_rope(q, pos, plan, out=q[:, :1].expand(4, 2, 64)),
                 lambda: sage.sage_rope(q[:0], pos[:0], plan)):
        with pytest.raises(sage.SageError):
            call()
