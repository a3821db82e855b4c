"""norm_rotate and norm_rotate_grads against their formulas in 64 bits.

Tolerances, in units u = 2^-24 of half a rounding in fp32.  A feature is x * inv * w: the sum of 128 squares has 8 additions in a
lane and 4 between lanes (relative 12 u, half of it in the root), root, division and two products: 12 u.  Cosine and sine: the
fraction of a turn is rounded once (2^-25 half turns, 1.6 u in the angle), the functions are good to 4 u: 6 u.  A turned feature
is two products and a sum of those: (12 + 6 + 3) u (|a| + |b|) magnitude, taken as 24 u.  bf16 outputs: half a step more, 2^-8."""
import itertools

import pytest
import torch

import paper_2502_08246_amd as saap

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
EPS = 1e-6


def _pairs(rot, pairs):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)


def _turned(y, positions, freqs, pairs, magnitude):
    """y [S,T,H,128] float64 -> turned, and |a| + |b| of every feature's pair."""
    a, b = _pairs(2 * freqs.numel(), pairs)
    angle = positions.double()[:, :, None, None] * freqs
    c, s = torch.cos(angle), torch.sin(angle)
    out, size = y.clone(), y.abs().clone()
    out[..., a] = magnitude * (y[..., a] * c - y[..., b] * s)
    out[..., b] = magnitude * (y[..., b] * c + y[..., a] * s)
    size[..., a] = size[..., b] = abs(magnitude) * (y[..., a].abs() + y[..., b].abs())
    return out, size


def _features(x, w, norm, eps=EPS):
    x = x.double()
    if not norm:
        return x
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return y if w is None else y * w.double()


def _inputs(S, T, Hq, Hkv, rot, dtype, seed, per_head=False, norm=True, fused=True, far=0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    if fused:
        rows = rand(S, T, (Hq + 2 * Hkv) * 128).to(dtype).to(DEV)
        q, k = rows[..., :Hq * 128].unflatten(2, (Hq, 128)), rows[..., Hq * 128:(Hq + Hkv) * 128].unflatten(2, (Hkv, 128))
    else:
        q, k = rand(S, T, Hq, 128).to(dtype).to(DEV), rand(S, T, Hkv, 128).to(dtype).to(DEV)
    positions = (torch.randint(0, 5000, (S, T), generator=g) + far).to(torch.int32)
    freqs = saap.rotary_frequencies(rot, device="cpu")
    qw, kw = (1 + 0.3 * rand(*((Hq, 128) if per_head else (128,))), 1 + 0.3 * rand(*((Hkv, 128) if per_head else (128,)))) if norm else (None, None)
    return q, k, positions, freqs, qw, kw


def _near(got, want, size, what):
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    err = (got.cpu().double() - want).abs()
    bad = err > 24 * U * size + half * want.abs() * (1 + 1e-3)
    assert not bad.any(), f"{what}: {int(bad.sum())} off, worst {float((err / (size + 1e-30)).max()):.3e}"


def _dev(t):
    return None if t is None else t.to(DEV)


SHAPES = [(1, 1, 32, 8), (3, 1, 4, 1), (2, 7, 1, 1), (1, 65, 2, 2), (2, 130, 8, 4), (5, 3, 6, 2), (1, 1001, 3, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("S,T,Hq,Hkv", SHAPES)
def test_forward(S, T, Hq, Hkv, pairs, dtype):
    for n, (rot, per_head, fused) in enumerate([(128, False, True), (64, True, False), (96, True, True), (16, False, False)]):
        q, k, positions, freqs, qw, kw = _inputs(S, T, Hq, Hkv, rot, dtype, 10 * n + T, per_head, True, fused)
        mag = 1.0 + 0.25 * n
        q_rot, q_feat, k_rot, k_feat = saap.norm_rotate(q, k, _dev(positions), _dev(freqs), _dev(qw), _dev(kw), eps=EPS, pairs=pairs, magnitude=mag)
        assert q_rot.shape == q_feat.shape == (S, T, Hq, 128) and k_rot.shape == k_feat.shape == (S, Hkv, T, 128)
        for x, w, feat, rotated in ((q, qw, q_feat, q_rot), (k, kw, k_feat.transpose(1, 2), k_rot.transpose(1, 2))):
            y = _features(x.cpu(), w, True)
            want, size = _turned(y, positions, freqs, pairs, mag)
            _near(feat, y, y.abs(), f"features rot={rot}")
            _near(rotated, want, size, f"rotated rot={rot}")


@pytest.mark.parametrize("pairs", [False, True])
def test_without_norm_features_are_the_input_and_far_positions_are_turned_exactly(pairs):
    q, k, positions, freqs, _, _ = _inputs(2, 33, 4, 2, 128, torch.float32, 3, norm=False, far=2 ** 31 - 6000)
    q_rot, q_feat, k_rot, k_feat = saap.norm_rotate(q, k, _dev(positions), _dev(freqs), norm=False, pairs=pairs)
    assert torch.equal(q_feat, q) and torch.equal(k_feat, k.transpose(1, 2))
    want, size = _turned(q.cpu().double(), positions, freqs, pairs, 1.0)
    _near(q_rot, want, size, "far positions")
    # negative ones turn the other way
    back, _, _, _ = saap.norm_rotate(q, None, -_dev(positions), _dev(freqs), norm=False, pairs=pairs)
    want, size = _turned(q.cpu().double(), -positions, freqs, pairs, 1.0)
    _near(back, want, size, "negative positions")


def test_one_tensor_outputs_passed_in_and_what_is_not_asked_for():
    q, k, positions, freqs, qw, kw = _inputs(2, 9, 4, 2, 128, torch.bfloat16, 4)
    pos, f = _dev(positions), _dev(freqs)
    whole = saap.norm_rotate(q, k, pos, f, _dev(qw), _dev(kw))
    only_q = saap.norm_rotate(q, None, pos, f, _dev(qw), q_features=False)
    assert only_q[1:] == (None, None, None) and torch.equal(only_q[0], whole[0])
    only_k = saap.norm_rotate(None, k, pos, f, k_weight=_dev(kw))
    assert only_k[:2] == (None, None) and torch.equal(only_k[2], whole[2]) and torch.equal(only_k[3], whole[3])
    out = torch.empty_like(whole[2])
    got = saap.norm_rotate(q, k, pos, f, _dev(qw), _dev(kw), q_features=False, k_features=False, k_rot=out)
    assert got[2] is out and got[1] is None and got[3] is None and torch.equal(out, whole[2])


def test_rows_that_are_no_numbers_stay_in_their_rows():
    q, k, positions, freqs, qw, kw = _inputs(1, 20, 4, 4, 64, torch.float32, 5)
    want = saap.norm_rotate(q, k, _dev(positions), _dev(freqs), _dev(qw), _dev(kw))
    q2 = q.clone()
    q2[0, 3, 1, 5] = float("nan")
    q2[0, 7, 2, 100] = float("inf")
    q2[0, 9, 0] = 0.0
    got = saap.norm_rotate(q2, k, _dev(positions), _dev(freqs), _dev(qw), _dev(kw))
    other = torch.ones(1, 20, 4, dtype=torch.bool, device=DEV)
    other[0, 3, 1] = other[0, 7, 2] = other[0, 9, 0] = False
    for i in (0, 1):
        assert torch.equal(got[i][other], want[i][other])
        assert got[i][0, 3, 1].isnan().all() and (got[i][0, 9, 0] == 0).all()
    assert torch.equal(got[2], want[2])


def _grads_reference(x, positions, freqs, pairs, mag, w, g_rot, g_feat, norm):
    """By autograd on the formula in 64 bits; and the sizes that its rounding errors are measured by."""
    x = x.double().requires_grad_(True)
    w = None if w is None else w.double().requires_grad_(True)
    y = _features(x, w, norm)
    turned, _ = _turned(y, positions, freqs, pairs, mag)
    loss = 0.0
    if g_rot is not None:
        loss = loss + (turned * g_rot.double()).sum()
    if g_feat is not None:
        loss = loss + (y * g_feat.double()).sum()
    got = torch.autograd.grad(loss, [x] if w is None else [x, w])
    with torch.no_grad():
        size = torch.zeros_like(y)
        if g_rot is not None:
            _, size = _turned(g_rot.double(), -positions, freqs, pairs, mag)
        if g_feat is not None:
            size = size + g_feat.double().abs()
        if not norm:
            return got[0], None, size, None
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
        n = (x * r).abs()
        u = size if w is None else size * w.abs()
        dx_size = r * (u + n * (u * n).mean(-1, keepdim=True))
        dw_size = None if w is None else (size * n).sum((0, 1) if w.dim() == 2 else (0, 1, 2))
    return got[0], None if w is None else got[1], dx_size, dw_size


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S,T,Hq,Hkv", SHAPES + [(4, 700, 4, 2)])
def test_gradients(S, T, Hq, Hkv, dtype):
    """dx: the turned gradient's 24 u, the mean over 128 products (12 u) and six more roundings: 48 u of its size, which _near
    reads as twice 24.  dweight: R rows are added up, (R + 48) u of the sum of sizes at worst."""
    for n, (rot, pairs, per_head, norm, feat, fused) in enumerate(itertools.islice(itertools.cycle([
            (128, False, False, True, True, True), (64, True, True, True, False, False), (32, False, True, True, True, True),
            (128, True, False, False, True, False)]), 4)):
        q, k, positions, freqs, qw, kw = _inputs(S, T, Hq, Hkv, rot, dtype, 7 * n + S, per_head, norm, fused)
        g = torch.Generator().manual_seed(n)
        rand = lambda *s: torch.randn(*s, generator=g).to(dtype).to(DEV)  # noqa: E731
        g_q_rot, g_k_rot = rand(S, T, Hq, 128), rand(S, Hkv, T, 128)
        g_q_feat, g_k_feat = (rand(S, T, Hq, 128), rand(S, Hkv, T, 128)) if feat else (None, None)
        mag = 1.0 + 0.125 * n
        run = lambda: saap.norm_rotate_grads(q, k, _dev(positions), _dev(freqs), g_q_rot, g_q_feat, g_k_rot, g_k_feat, _dev(qw), _dev(kw),  # noqa: E731
                                             norm=norm, eps=EPS, pairs=pairs, magnitude=mag)
        got = run()
        again = run()
        for a, b in zip(got, again):
            assert (a is None and b is None) or torch.equal(a, b)
        heads = lambda t: None if t is None else t.transpose(1, 2).cpu()  # noqa: E731
        for x, w, gr, gf, dx, dw in ((q, qw, g_q_rot.cpu(), None if g_q_feat is None else g_q_feat.cpu(), got[0], got[2]),
                                     (k, kw, heads(g_k_rot), heads(g_k_feat), got[1], got[3])):
            want, want_w, size, size_w = _grads_reference(x.cpu(), positions, freqs, pairs, mag, w, gr, gf, norm)
            _near(dx, want, 2 * size, f"dx case {n}")
            if w is None:
                assert dw is None
            else:
                rows = S * T * (1 if per_head else x.shape[2])
                err = (dw.cpu().double() - want_w).abs()
                assert (err <= (rows + 48) * U * size_w).all(), f"dweight case {n}: {float((err / size_w).max()):.3e}"


def test_gradients_by_differences():
    """A central difference of the fp32 forward pass: its step of 2^-7 is exact in x, the third derivative and the rounding of
    two sums of 8 * 128 outputs leave some 2^-11 of the sum's size."""
    q, _, positions, freqs, qw, _ = _inputs(1, 2, 4, 1, 64, torch.float32, 11, fused=False)
    g = torch.randn(1, 2, 4, 128, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    dq, _, dw, _ = saap.norm_rotate_grads(q, None, _dev(positions), _dev(freqs), g, g, None, None, _dev(qw))
    def loss(x, w):
        rotated, feat, _, _ = saap.norm_rotate(x, None, _dev(positions), _dev(freqs), w)
        return float((g.double() * (rotated.double() + feat.double())).sum())
    h = 2.0 ** -7
    for at in [(0, 0, 0, 3), (0, 1, 2, 40), (0, 1, 3, 127)]:
        up, down = q.clone(), q.clone()
        up[at] += h
        down[at] -= h
        slope = (loss(up, _dev(qw)) - loss(down, _dev(qw))) / float(up[at] - down[at])
        assert abs(slope - float(dq[at])) <= 2.0 ** -11 * 8, (at, slope, float(dq[at]))
    for f in (0, 63, 100):
        up, down = _dev(qw).clone(), _dev(qw).clone()
        up[f] += h
        down[f] -= h
        slope = (loss(q, up) - loss(q, down)) / float(up[f] - down[f])
        assert abs(slope - float(dw[f])) <= 2.0 ** -11 * 8, (f, slope, float(dw[f]))


def test_captured_and_on_two_streams():
    q, k, positions, freqs, qw, kw = _inputs(2, 300, 8, 2, 128, torch.bfloat16, 12)
    pos, f, qw, kw = _dev(positions), _dev(freqs), _dev(qw), _dev(kw)
    g = torch.randn(2, 300, 8, 128, device=DEV).to(torch.bfloat16)
    gk = torch.randn(2, 2, 300, 128, device=DEV).to(torch.bfloat16)
    both = lambda: saap.norm_rotate(q, k, pos, f, qw, kw) + saap.norm_rotate_grads(q, k, pos, f, g, None, gk, gk, qw, kw)  # noqa: E731
    want = both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = both()
    here = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, here, there))


def test_tokens_far_apart():
    """Rows 2^30 elements apart, the last one 4 GB and more behind the first: each has the bits that it has in a dense tensor."""
    g = torch.Generator().manual_seed(31)
    wide = torch.zeros(1, 4, 2 ** 30, dtype=torch.bfloat16, device=DEV)
    wide[0, :, :6 * 128] = torch.randn(4, 6 * 128, generator=g).to(torch.bfloat16).to(DEV)
    q, k = wide[..., :4 * 128].unflatten(2, (4, 128)), wide[..., 4 * 128:6 * 128].unflatten(2, (2, 128))
    pos, f, w = torch.arange(4, dtype=torch.int32, device=DEV)[None], saap.rotary_frequencies(128, device=DEV), torch.rand(128, generator=g).to(DEV)
    far, near = saap.norm_rotate(q, k, pos, f, w, w), saap.norm_rotate(q.contiguous(), k.contiguous(), pos, f, w, w)
    assert all(torch.equal(a, b) for a, b in zip(far, near))
    grads = [torch.randn(t.shape, generator=g).to(torch.bfloat16).to(DEV) for t in near]
    far, near = (saap.norm_rotate_grads(a, b, pos, f, *grads, w, w) for a, b in ((q, k), (q.contiguous(), k.contiguous())))
    assert all(torch.equal(a, b) for a, b in zip(far, near))
