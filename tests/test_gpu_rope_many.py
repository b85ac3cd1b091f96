"""Rotary positions of so many tokens that a wavefront takes several heads of a token, one after the other, with the angles of the first."""
import pytest
import torch

import paper_2505_21136_amd as sage
from test_gpu_rope import DEV, _check, _want

pytestmark = pytest.mark.gpu


def _steps(T, H, d):
    """Heads that a lane takes: as many as there are for its place in a wavefront, if that leaves eight wavefronts to each SIMD of 256 CUs."""
    rows = 1024 // d
    return min(-(-H // rows), max(1, -(-T * H // rows) // (8 * 4 * 256)))


@pytest.mark.parametrize("T,Hq,Hkv,d,steps", [(16411, 32, 8, 128, 5), (16411, 31, 8, 128, 5), (9001, 33, 4, 128, 5), (4500, 24, 8, 128, 2), (16411, 37, 3, 64, 3),
                                              (16411, 13, 3, 128, 2), (40003, 5, 0, 128, 1), (14000, 29, 2, 64, 2)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_several_heads_a_wavefront(T, Hq, Hkv, d, steps, layout):
    assert _steps(T, Hq + Hkv, d) == steps
    g = torch.Generator().manual_seed(T + Hq)
    plan = sage.rope_plan(d - 32, layout=layout, scaling="yarn", factor=4.0, trained_len=4096)
    qkv = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16).to(DEV)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv] if Hkv else None
    pos = torch.randint(-1 << 20, 1 << 20, (T,), generator=g).to(torch.int32)
    got = sage.sage_rope(q, pos.to(DEV), plan, k=k)
    pick = torch.cat([torch.randperm(T, generator=g)[:150], torch.arange(40), torch.arange(T - 40, T)])
    for y, x, name in zip(got if Hkv else (got,), (q, k), "qk"):
        _check(y[pick.to(DEV)], *_want(x[pick.to(DEV)], pos[pick], plan), torch.bfloat16, name)
    # and all of them: a token by itself is rotated the same, bit for bit
    for a in range(0, T, 1000):
        part = sage.sage_rope(q[a:a + 1000], pos[a:a + 1000].to(DEV), plan, k=None if k is None else k[a:a + 1000])
        for y, x in zip(got if Hkv else (got,), part if Hkv else (part,)):
            assert torch.equal(y[a:a + 1000], x), a
    # in place
    sage.sage_rope(q, pos.to(DEV), plan, k=k, out=q, k_out=k)
    assert torch.equal(q, got[0] if Hkv else got) and (k is None or torch.equal(k, got[1]))
