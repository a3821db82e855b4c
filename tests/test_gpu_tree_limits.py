"""tree_decode_attention where its work is split differently: many units, lists around the length that a wave holds, rows of several
waves and workgroups, values that are no numbers on every way through, and the largest caches.  Tolerances: test_gpu_tree.py."""
import math

import pytest
import torch

import paper_2502_08246_amd as saap
from test_gpu_tree import DEV, SCALE, U, Case, _check, _slopes

pytestmark = pytest.mark.gpu


def _compare_all(c, got, lse, seen, scale=SCALE, out_bf16=False):
    """The definition for all sequences and heads together (no caps, no biases)."""
    S, T, Hq, Hkv, N = c.S, c.T, c.Hq, c.Hkv, c.N
    G = Hq // Hkv
    q = c.q.double().view(S, T, Hkv, G, 128).permute(0, 2, 1, 3, 4).reshape(S * Hkv, T * G, 128)
    k = torch.cat((c.K_held.double(), c.kt.double()), 2).view(S * Hkv, N + T, 128)
    v = torch.cat((c.V_held.double(), c.vt.double()), 2).view(S * Hkv, N + T, 128)
    drafted = ((c.tree[:, :, None] >> torch.arange(T)) & 1).bool()[:, None].expand(S, Hkv, T, T)
    see = torch.cat((seen, drafted), 3).reshape(S * Hkv, T, 1, N + T).expand(-1, -1, G, -1).reshape(S * Hkv, T * G, N + T)
    a = q @ k.transpose(1, 2) * scale
    delta = (130 * U * abs(scale) * (q.abs() @ k.abs().transpose(1, 2)) + 8 * U * a.abs()).masked_fill(~see, 0.0).amax(2)
    a = a.masked_fill(~see, -math.inf)
    count, top = see.sum(2), a.amax(2)
    p = torch.exp(a - top.masked_fill(count == 0, 0.0)[..., None])
    total = p.sum(2)
    p = p / total.clamp(min=1e-300)[..., None]
    back = lambda x: x.view(S, Hkv, T, G, -1).permute(0, 2, 1, 3, 4).reshape(S, T, Hq, -1)  # noqa: E731
    want_lse = top.masked_fill(count == 0, 0.0) + torch.log(total)
    rel = 2.2 * delta + (count + 64) * U + (2.0 ** -16 if out_bf16 else 0.0)
    _check(got, back(p @ v), back(rel[..., None] * (p @ v.abs())), "out")
    _check(lse, back(want_lse)[..., 0], back(delta + (count + 64) * U + 4 * U * want_lse.abs().nan_to_num(posinf=0.0))[..., 0], "lse")


UNITS = [("bf16", 40, 1, 8, 2, 300, "none"), ("f32", 65, 3, 4, 1, 130, "none"), ("bf16", 130, 2, 8, 4, 60, "none"),
         ("fp8", 520, 1, 4, 1, 70, "none"), ("bf16", 1024, 1, 4, 4, 40, "none"), ("bf16", 150, 17, 4, 2, 50, "none"),
         ("f32", 300, 9, 8, 1, 40, "none"), ("bf16", 66, 3, 8, 2, 200, "own"), ("f32", 300, 2, 2, 2, 50, "own"), ("bf16", 520, 1, 4, 1, 60, "shared"),
         ("fp8", 150, 9, 8, 2, 60, "own"), ("bf16", 300, 12, 4, 1, 60, "shared")]


@pytest.mark.parametrize("dtype,S,T,Hq,Hkv,N,lists", UNITS)
def test_many_sequences(dtype, S, T, Hq, Hkv, N, lists):
    """Fewer shares than units, or a few to each; lengths from none to all of the keys."""
    c = Case(dtype, S, T, Hq, Hkv, N, 16, 3, lists, (2, 10) if lists == "own" else None, seed=S, ragged=lists == "none").cache()
    for out in (torch.float32, torch.bfloat16):
        _compare_all(c, *c.run(out), c.seen, out_bf16=out == torch.bfloat16)


def test_one_length_and_more_units_than_shares():
    c = Case("bf16", 257, 6, 16, 4, 90, seed=2).cache()
    _compare_all(c, *c.run(), c.seen)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("nprobe,window", [(61, (1, 20)), (62, (1, 20)), (63, None), (63, (1, 20)), (64, None), (1, None)])
@pytest.mark.parametrize("T", [1, 4, 16])
def test_lists_about_as_long_as_a_wave_is_wide(dtype, nprobe, window, T):
    c = Case(dtype, 2, T, 8, 2, 1500, 256, nprobe, "shared", window, seed=nprobe).cache()
    _compare_all(c, *c.run(), c.seen)
    # ids that are none, and ids listed twice
    if nprobe > 8:
        sel = c.sel.clone()
        sel[..., 1], sel[..., 4], sel[..., -1] = -1, 256 + bool(window), 2 ** 31 - 1
        sel[0, 1, 5] = sel[0, 1, 0]
        sel[1, 0, 7] = sel[1, 0, 6] = sel[1, 0, -2]
        if window:
            sel[..., 2] = 256                            # the resident run itself
        c.sel = sel
        member = torch.zeros(2, 2, 258, dtype=torch.bool)
        member.scatter_(-1, sel.long().where((sel >= 0) & (sel < 256), torch.tensor(257)), True)
        c.seen = member.gather(2, c.ids.long())[:, :, None].expand(-1, -1, T, -1)
        if window:
            c.seen = c.seen | (c.kpos < 1) | (c.kpos >= 1500 - 20)
        _compare_all(c, *c.run(), c.seen)


ROWS = [(9, 4, 1), (33, 1, 1), (16, 8, 1), (20, 4, 1), (33, 4, 1), (33, 8, 1), (64, 8, 2), (64, 4, 1)]   # T, G, Hkv


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("T,G,Hkv", ROWS)
@pytest.mark.parametrize("lists", ["none", "own", "shared"])
def test_rows_of_several_waves(dtype, T, G, Hkv, lists):
    c = Case(dtype, 2, T, G * Hkv, Hkv, 1200, 64, 9, lists, (1, 40) if lists == "own" else None, seed=T * G, ragged=lists == "none").cache()
    for out in (torch.float32, torch.bfloat16):
        _compare_all(c, *c.run(out), c.seen, out_bf16=out == torch.bfloat16)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("T,G", [(12, 4), (33, 2), (20, 8)])
@pytest.mark.parametrize("lists", ["none", "own"])
def test_rows_of_several_waves_with_shaped_scores(dtype, T, G, lists):
    c = Case(dtype, 1, T, G, 1, 400, 32, 6, lists, (1, 30) if lists == "own" else None, seed=T).cache()
    starts = torch.randint(0, 450, (1, T), generator=c.g).to(torch.int32)
    c.compare(softcap=4.0, slopes=_slopes(G), starts=starts)
    c.compare(torch.bfloat16, slopes=-_slopes(G))


def _slot(c, s, h, position):
    """Where the cache holds a key."""
    if c.lists == "none":
        return position
    off, ln, idx = c.off[s, h].tolist(), c.ln[s, h].tolist(), c.idx[s, h].tolist()
    return next(at for b in range(len(ln)) for at in range(off[b], off[b] + ln[b]) if idx[at] == position)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("T,G", [(1, 4), (2, 4), (8, 4), (12, 4), (40, 4)])
@pytest.mark.parametrize("lists", ["none", "shared", "own"])
def test_values_that_are_no_numbers(dtype, T, G, lists):
    """An infinity among the values makes that feature infinite in the rows that attend it and in no other; a NaN among the keys makes
    its rows NaN."""
    c = Case(dtype, 2, T, 2 * G, 2, 300, 16, 5, lists, seed=T, ragged=False).cache()
    starts = torch.randint(0, 300, (2, T), generator=c.g).to(torch.int32)
    code = dtype == "fp8"                                # E4M3 has no infinities
    bad = float("nan") if code else float("inf")
    at = _slot(c, 1, 0, 150)
    c.Vd[1, 0, at, 9] = 0x7f if code else bad
    c.V_held = c.V_held.clone()
    c.V_held[1, 0, 150, 9] = bad
    c.compare()
    c.compare(starts=starts)
    c.compare(drafts=False)
    if T > 1:
        c.vt[0, 1, 1, 3] = -float("inf")
        c.compare(torch.bfloat16)
    at = _slot(c, 0, 1, 222)
    c.Kd[0, 1, at, 0] = 0x7f if code else float("nan")
    c.K_held = c.K_held.clone()
    c.K_held[0, 1, 222, 0] = float("nan")
    c.compare()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("scale", [0.0, -0.05])
@pytest.mark.parametrize("T", [2, 20])
def test_scales_that_are_not_positive(dtype, scale, T):
    c = Case(dtype, 1, T, 4, 1, 200, seed=T).cache()
    f = saap.dense_tree_decode_attention_fp8 if c.scales else saap.dense_tree_decode_attention
    got, lse = f(c.q.to(DEV), c.Kd, c.Vd, *c.scales, scale, c.kt.to(DEV), c.vt.to(DEV), c.tree.to(DEV), out_dtype=torch.float32)
    _compare_all(c, got, lse, c.seen, scale)


@pytest.mark.parametrize("T", [1, 30])
def test_nothing_to_attend(T):
    """No listed key and no drafted one, in some sequences or all: zeros and -inf; what the empty cache holds does not matter."""
    for dtype in ("bf16", "f32", "fp8"):
        c = Case(dtype, 3, T, 4, 2, 64, seed=1).cache()
        c.Kd[:] = 0x7f if dtype == "fp8" else float("nan")
        c.Vd[:] = 0x7f if dtype == "fp8" else float("nan")
        c.n_keys = torch.tensor([0, -5, 0], dtype=torch.int32)
        got, lse = c.run(drafts=False)
        assert (got == 0).all() and (lse == -math.inf).all()
        c.tree[1] = 0
        got, lse = c.run()
        assert (got[1] == 0).all() and (lse[1] == -math.inf).all() and torch.isfinite(got).all()
        c = Case(dtype, 2, T, 4, 2, 64, 16, 0, "shared", seed=1).cache()
        c.sel = torch.full((2, 2, 4), -1, dtype=torch.int32)
        got, lse = c.run(drafts=False)
        assert (got == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("T", [2, 16])
def test_the_end_of_the_longest_cache(T):
    """Rows that begin 4 GB into the cache: starts leave the last keys, values before them would show."""
    N, last = (1 << 23) - 1, 200
    K, V = torch.zeros(1, 1, N, 128, device=DEV), torch.ones(1, 1, N, 128, device=DEV)
    c = Case("f32", 1, T, 4, 1, last, seed=3)
    K[0, 0, -last:], V[0, 0, -last:] = c.K[0, 0].to(DEV), c.V[0, 0].to(DEV)
    c.K_held, c.V_held = c.K, c.V
    starts = torch.full((1, T), N - last, dtype=torch.int32, device=DEV)
    got, lse = saap.dense_tree_decode_attention(c.q.to(DEV), K, V, SCALE, c.kt.to(DEV), c.vt.to(DEV), c.tree.to(DEV), starts=starts,
                                                out_dtype=torch.float32)
    _compare_all(c, got, lse, c.seen)


def test_sequences_of_a_batch_do_not_change_each_other():
    """A sequence decoded alone, among others, and captured with them."""
    c = Case("bf16", 5, 6, 8, 2, 700, ragged=True, seed=21).cache()
    d = lambda x: x.to(DEV)  # noqa: E731
    args = [d(c.q), c.Kd, c.Vd, SCALE, d(c.kt), d(c.vt), d(c.tree)]
    n = d(c.n_keys)
    whole = saap.dense_tree_decode_attention(*args, n_keys=n)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = saap.dense_tree_decode_attention(*args, n_keys=n)
    for lengths in (c.n_keys, torch.zeros(5, dtype=torch.int32), torch.tensor([700, 1, 0, 33, 699], dtype=torch.int32)):
        n.copy_(lengths)
        graph.replay()
        eager = saap.dense_tree_decode_attention(*args, n_keys=n)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        for s in (0, 3):
            one = [x[s:s + 1] if torch.is_tensor(x) else x for x in args]
            got, lse = saap.dense_tree_decode_attention(*one, n_keys=n[s:s + 1])
            assert torch.allclose(got[0], eager[0][s], rtol=1e-4, atol=2e-5) and torch.allclose(lse[0], eager[1][s], rtol=1e-5, atol=1e-5)
    assert torch.isfinite(whole[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("T", [2, 12, 40])
@pytest.mark.parametrize("lists", ["none", "shared", "own"])
def test_queries_of_tokens_that_are_not_there(dtype, T, lists):
    """A padded batch whose padding is NaN or infinite: those tokens' rows alone are no numbers, also where a value is infinite too."""
    c = Case(dtype, 2, T, 4, 2, 300, 16, 5, lists, seed=T + 1).cache()
    c.vt[0, 0, 0, 5] = float("inf")
    c.tree[:, :T - 1] |= 1
    c.tree[:, T - 1] = 0
    c.q[0, T - 1] = float("nan")
    c.q[1, T - 1, 2] = float("inf")
    c.q[1, T - 1, 2, ::2] = -float("inf")
    got, lse = c.run()
    seen = c.seen[:, :, T - 1].any(-1)                   # [S,Hkv]
    assert seen.all()
    assert got[0, T - 1].isnan().all() and lse[0, T - 1].isnan().all()
    c.q[0, T - 1] = 0
    c.q[1, T - 1, 2] = 0
    want, want_lse = c.run()
    assert torch.equal(got[:, :T - 1], want[:, :T - 1]) and torch.equal(lse[:, :T - 1], want_lse[:, :T - 1])
    rest = [h for h in range(4) if h != 2]
    assert torch.equal(got[1, T - 1, rest], want[1, T - 1, rest])
    c.compare()


@pytest.mark.parametrize("T", [1, 3, 20])
def test_any_run_may_be_the_resident_one(T):
    """Among the listed ones of some tokens, the first, the last, and where nothing else is listed."""
    for nprobe in (0, 4, 70):
        for run in (0, 7, 127):
            c = Case("bf16", 2, T, 4, 1, 900, 128, nprobe, "own", seed=run).cache()
            if nprobe:
                c.sel[0, 0, 0, 1] = run
                member = torch.zeros(2, T, 1, 128, dtype=torch.bool).scatter_(-1, c.sel.long(), True).transpose(1, 2)
                c.seen = member.gather(3, c.ids.long()[:, :, None].expand(-1, -1, T, -1))
            c.seen = c.seen | (c.ids == run)[:, :, None]
            d = lambda x: x.to(DEV)  # noqa: E731
            got, lse = saap.tree_decode_attention(d(c.q), c.Kd, c.Vd, c.off, c.ln, d(c.sel), SCALE, d(c.kt), d(c.vt), d(c.tree), resident_run=run,
                                                  out_dtype=torch.float32)
            _compare_all(c, got, lse, c.seen)


def test_lengths_outside_the_cache_are_cut():
    c = Case("bf16", 3, 4, 4, 2, 100, seed=4).cache()
    c.n_keys = torch.tensor([101, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    got, lse = c.run()
    c.seen = c.seen.clone()
    c.seen[2] = False
    _compare_all(c, got, lse, c.seen)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_few_rows_captured_and_replayed(dtype):
    """Shares that the last workgroup of a unit adds up: counters are back at zero after every call, on its own and in a graph that
    replays with other lists, other calls between."""
    c = Case(dtype, 2, 2, 8, 2, 3000, 64, 20, "shared", (1, 50), seed=5).cache()
    d = lambda x: x.to(DEV)  # noqa: E731
    f = saap.tree_decode_attention_fp8 if c.scales else saap.tree_decode_attention
    sel = d(c.sel)
    args = (d(c.q), c.Kd, c.Vd, *c.scales, c.off, c.ln, sel, SCALE, d(c.kt), d(c.vt), d(c.tree))
    call = lambda: f(*args, resident_run=64, out_dtype=torch.float32)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call() + call()
    for i in range(4):
        sel.copy_(torch.rand(2, 2, 64, generator=c.g).topk(20, -1).indices.to(torch.int32))
        graph.replay()
        eager = call()
        torch.cuda.synchronize()
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])
        assert torch.equal(out[2], eager[0]) and torch.equal(out[3], eager[1])
    c.sel = sel.cpu()
    member = torch.zeros(2, 2, 64, dtype=torch.bool).scatter_(-1, c.sel.long(), True)
    seen = member.gather(2, c.ids.long())[:, :, None].expand(-1, -1, 2, -1)
    _compare_all(c, *eager, seen | (c.kpos < 1) | (c.kpos >= 2950))
