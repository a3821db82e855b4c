"""The gradients of norm_rotate's weights over many rows: their sums lose nothing however many rows there are.

u = 2^-24.  Four rows are added in fp32: of equal terms t the sums 2t, 3t and 4t are off by at most 2 u, 2 u and 4 u of t (half a step
between 2 and 4, and from 4 on), together 2 u of 4t.  Those are added in double, a workgroup's sum is rounded (u), and so is the
result (u): 4 u of the sum of the sizes of terms that are alike; of any terms, whose partial sums are no larger than the sum of
sizes, 3 additions of u, and 2: 5 u.  In the first test x is plus or minus one everywhere and eps is 0, so that every norm is 1 and a
row adds its gradient of the features, times that sign: the scale 1 / sqrt(mean) is within 2 u of 1, 6 u in all.  In the second
every term has the forward call's 12 u (sum of squares, root, product), with a sum's 5 u: below 40 u."""
import pytest
import torch

import paper_2502_08246_amd as saap

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
SHAPES = [(1, 100003, 1, 0), (2, 30001, 4, 2), (1, 65537, 2, 2), (1, 40000, 0, 1)]


def _both(S, T, Hq, Hkv, make):
    q = make(S, T, Hq) if Hq else None
    k = make(S, T, Hkv) if Hkv else None
    return q, k


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("S,T,Hq,Hkv", SHAPES)
def test_rows_that_are_all_rounded_the_same_way(S, T, Hq, Hkv, per_head):
    """Feature f of every gradient is 1 + 0.99 * 2^-(12 + f % 12): in fp32 a sum of such numbers that has grown to a power of two
    loses nearly half a step with every one."""
    g = torch.Generator(device=DEV).manual_seed(T)
    sign = lambda S, T, H: torch.randint(0, 2, (S, T, H, 128), generator=g, device=DEV).float() * 2 - 1  # noqa: E731
    q, k = _both(S, T, Hq, Hkv, sign)
    each = (1 + 0.99 * torch.exp2(-12.0 - torch.arange(128, device=DEV) % 12)).float()
    ones = lambda H: torch.ones((H, 128) if per_head else (128,), device=DEV)  # noqa: E731
    g_q = None if q is None else q * each
    g_k = None if k is None else (k * each).transpose(1, 2).contiguous()
    pos, freqs = torch.zeros(S, T, dtype=torch.int32, device=DEV), saap.rotary_frequencies(128, device=DEV)
    got = saap.norm_rotate_grads(q, k, pos, freqs, None, g_q, None, g_k, ones(Hq) if Hq else None, ones(Hkv) if Hkv else None, eps=0.0)
    for x, dw, H in ((q, got[2], Hq), (k, got[3], Hkv)):
        if x is None:
            assert dw is None
            continue
        want = each.double() * (S * T * (1 if per_head else H))
        off = ((dw.double() - want).abs() / want).max()
        assert float(off) <= 6 * U, f"{float(off) / U:.1f} u"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S,T,Hq,Hkv", SHAPES)
def test_many_rows(S, T, Hq, Hkv, dtype):
    g = torch.Generator(device=DEV).manual_seed(T + 1)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    q, k = _both(S, T, Hq, Hkv, lambda *s: rand(*s, 128).to(dtype))
    g_q = None if q is None else (rand(*q.shape) + 0.5 * q.float()).to(dtype)
    g_k = None if k is None else (rand(*k.shape) + 0.5 * k.float()).to(dtype)
    w = 1 + 0.2 * rand(128)
    pos = torch.arange(S * T, device=DEV, dtype=torch.int32).view(S, T)
    heads = lambda t: None if t is None else t.transpose(1, 2).contiguous()  # noqa: E731
    got = saap.norm_rotate_grads(q, k, pos, saap.rotary_frequencies(128, device=DEV), None, g_q, None, heads(g_k), w if Hq else None,
                                 w if Hkv else None)
    again = saap.norm_rotate_grads(q, k, pos, saap.rotary_frequencies(128, device=DEV), None, g_q, None, heads(g_k), w if Hq else None,
                                   w if Hkv else None)
    for x, gx, dw, dw2 in ((q, g_q, got[2], again[2]), (k, g_k, got[3], again[3])):
        if x is None:
            continue
        n = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
        each = gx.double() * n
        err = (dw.double() - each.sum((0, 1, 2))).abs()
        assert (err <= 40 * U * each.abs().sum((0, 1, 2))).all(), float((err / each.abs().sum((0, 1, 2))).max() / U)
        assert torch.equal(dw, dw2)
