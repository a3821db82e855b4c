"""tree_decode_attention and its dense and 8-bit forms against the definition in 64 bits, made of positions, bucket ids and lists
(no index).

Tolerances, u = 2^-24.  A score is a sum of 128 products: off by at most d = 130 u scale sum |q k|, plus 8 u of its size (scale,
cap) and 4 u of its bias; weights are off by e^2d - 1 in proportion and by the roundings of sums over N keys, (N + 64) u; in bf16
outputs a weight has 16 bits (2^-16) and the result half a step (2^-8).  All of it times sum p |v|."""
import math

import pytest
import torch

import paper_2502_08246_amd as saap

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
SCALE = 1.0 / math.sqrt(128)


def _tree(g, S, T, padded=True):
    parents = torch.full((S, T), -1, dtype=torch.int64)
    for t in range(1, T):
        parents[:, t] = torch.randint(-1, t, (S,), generator=g)
    if padded and T > 2:
        for s in range(S):
            n = int(torch.randint(T // 2 + 1, T + 1, (1,), generator=g))
            parents[s, n:] = T
    return saap.tree_masks(parents), parents


def _depth(parents):
    S, T = parents.shape
    d = torch.zeros(S, T, dtype=torch.int64)
    for s in range(S):
        for t in range(T):
            p = int(parents[s, t])
            d[s, t] = d[s, p] + 1 if 0 <= p < T else 0
    return d


def _fp8(x):
    scale = torch.exp2(torch.ceil(torch.log2(x.float().abs().amax((2, 3)).clamp(min=1e-30) / 448.0)))
    codes = (x.float() / scale[:, :, None, None]).to(torch.float8_e4m3fn)
    return codes, scale, codes.float() * scale[:, :, None, None]


def reference(q, K, V, seen, kt, vt, tree, scale, softcap=0.0, slopes=None, pos=None, kpos=None, out_bf16=False):
    """q [S,T,Hq,d], K, V [S,Hkv,N,d] as decoded, seen [S,Hkv,T,N], kpos [N].  -> out, lse, tolerances of both."""
    S, T, Hq, d = q.shape
    Hkv, N = K.shape[1:3]
    G = Hq // Hkv
    out, lse = torch.zeros(S, T, Hq, d, dtype=torch.float64), torch.zeros(S, T, Hq, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    q, K, V = q.double(), K.double(), V.double()
    for s in range(S):
        for h in range(Hkv):
            k, v = K[s, h], V[s, h]
            see = seen[s, h]
            if kt is not None:
                k, v = torch.cat((k, kt[s, h].double())), torch.cat((v, vt[s, h].double()))
                see = torch.cat((see, ((tree[s][:, None] >> torch.arange(T)) & 1).bool()), 1)
            for t in range(T):
                at = see[t].nonzero()[:, 0]
                for gg in range(G):
                    hq = h * G + gg
                    if at.numel() == 0:
                        lse[s, t, hq] = -math.inf
                        continue
                    qq = q[s, t, hq]
                    a = k[at] @ qq * scale
                    delta = 130 * U * scale * (k[at].abs() @ qq.abs()) + 8 * U * a.abs()
                    if softcap > 0:
                        a = softcap * torch.tanh(a / softcap)
                        delta = delta + 4 * U * softcap
                    if slopes is not None:
                        kp = kpos if kt is None else torch.cat((kpos, pos[s].long()))
                        bias = slopes[hq].double() * (pos[s, t].long() - kp[at]).double()
                        a = a - bias
                        delta = delta + 4 * U * (bias - bias.min()).abs()
                    top = a.max()
                    p = torch.exp(a - top)
                    lse[s, t, hq] = top + torch.log(p.sum())
                    p = p / p.sum()
                    out[s, t, hq] = p @ v[at]
                    rel = 2 * delta.max() * 1.1 + (at.numel() + 64) * U + (2.0 ** -16 if out_bf16 else 0.0)
                    # far keys: errors in their scores count by their weights
                    tol[s, t, hq] = rel * (p @ v[at].abs())
                    tol_lse[s, t, hq] = delta.max() + (at.numel() + 64) * U + 4 * U * lse[s, t, hq].abs()
    return out, lse, tol, tol_lse


def _check(got, want, tol, what):
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    got = got.cpu().double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), f"{what}: numbers where there should be none, or the other way"
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()])
    err = (got - want).abs()[fine]
    limit = (tol + half * want.abs() * (1 + 1e-3))[fine]
    assert (err <= limit).all(), f"{what}: off by up to {float((err / limit.clamp(min=1e-300)).max()):.2f} times the tolerance"


class Case:
    def __init__(self, dtype, S, T, Hq, Hkv, N, B=0, nprobe=0, lists="none", window=None, seed=0, ragged=False, slack=3):
        g = self.g = torch.Generator().manual_seed(seed * 101 + T)
        self.dtype, self.S, self.T, self.Hq, self.Hkv, self.N, self.B = dtype, S, T, Hq, Hkv, N, B
        row = torch.float32 if dtype == "f32" else torch.bfloat16
        rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.q, self.K, self.V = (1.5 * rand(S, T, Hq, 128)).to(row), (rand(S, Hkv, N, 128) + 0.5).to(row), rand(S, Hkv, N, 128).to(row)
        self.kt, self.vt = rand(S, Hkv, T, 128).to(row), rand(S, Hkv, T, 128).to(row)
        self.tree, parents = _tree(g, S, T)
        self.kpos = torch.arange(N)
        self.seen = torch.ones(S, Hkv, T, N, dtype=torch.bool)
        self.pos = (N + _depth(parents)).to(torch.int32)
        self.n_keys = None
        if ragged:
            self.n_keys = torch.randint(0, N + 1, (S,), generator=g).to(torch.int32)
            self.n_keys[0] = 0
            self.n_keys[-1] = N
            self.seen &= (self.kpos < self.n_keys[:, None, None, None])
        self.lists, self.window = lists, window
        if lists != "none":
            self.ids = torch.randint(0, B, (S, Hkv, N), generator=g).to(torch.int32)
            shape = (S, T, Hkv, B) if lists == "own" else (S, Hkv, B)
            self.sel = torch.rand(shape, generator=g).topk(nprobe, -1).indices.to(torch.int32) if nprobe else torch.zeros(*shape[:-1], 0, dtype=torch.int32)
            member = torch.zeros(*shape, dtype=torch.bool).scatter_(-1, self.sel.long(), True)
            member = member.transpose(1, 2) if lists == "own" else member[:, :, None].expand(-1, -1, T, -1)
            self.seen = member.gather(3, self.ids.long()[:, :, None].expand(-1, -1, T, -1))
            if window:
                sink, recent = window
                self.seen = self.seen | (self.kpos < sink) | (self.kpos >= N - recent)

    def cache(self, slack=3):
        """The call's arguments on the device, and the values as the cache holds them."""
        K, V = self.K.to(DEV), self.V.to(DEV)
        if self.lists != "none":
            ids = self.ids.to(DEV)
            if self.window:
                index = saap.build_windowed_index(ids, K, V, self.B, slack, *self.window)[:5]
            else:
                index = saap.build_bucket_index(ids, K, V, self.B, slack)
            self.off, self.ln, self.idx, K, V = index
        self.Kd, self.Vd, self.scales = K, V, ()
        if self.dtype == "fp8":
            kc, ks, _ = _fp8(K)
            vc, vs, _ = _fp8(V)
            self.Kd, self.Vd, self.scales = kc.view(torch.uint8), vc.view(torch.uint8), (ks, vs)
            decode = lambda x, s: (x.float().to(DEV) / s[:, :, None, None]).to(torch.float8_e4m3fn).float().mul(s[:, :, None, None]).cpu()  # noqa: E731
            self.K_held, self.V_held = decode(self.K, ks), decode(self.V, vs)
        else:
            self.K_held, self.V_held = self.K, self.V
        return self

    def run(self, out_dtype=torch.float32, drafts=True, **kw):
        d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        more = {n: d(t) if torch.is_tensor(t) else t for n, t in kw.items()}
        if drafts:
            more.update(k_tree=d(self.kt), v_tree=d(self.vt), tree=d(self.tree))
        if self.lists == "none":
            f = saap.dense_tree_decode_attention_fp8 if self.scales else saap.dense_tree_decode_attention
            return f(d(self.q), self.Kd, self.Vd, *self.scales, SCALE, n_keys=d(self.n_keys), out_dtype=out_dtype, **more)
        f = saap.tree_decode_attention_fp8 if self.scales else saap.tree_decode_attention
        return f(d(self.q), self.Kd, self.Vd, *self.scales, self.off, self.ln, d(self.sel), SCALE, idx=self.idx,
                 resident_run=self.B if self.window else -1, out_dtype=out_dtype, **more)

    def compare(self, out_dtype=torch.float32, drafts=True, softcap=0.0, slopes=None, starts=None):
        kw = dict(softcap=softcap)
        if slopes is not None:
            kw.update(slopes=slopes, pos=self.pos)
        seen = self.seen
        if starts is not None:
            kw["starts"] = starts
            seen = seen & (self.kpos >= starts.long()[:, None, :, None])
        got, lse = self.run(out_dtype, drafts, **kw)
        want, want_lse, tol, tol_lse = reference(self.q, self.K_held, self.V_held, seen, self.kt if drafts else None, self.vt, self.tree, SCALE,
                                                 softcap, slopes, self.pos, self.kpos, out_dtype == torch.bfloat16)
        _check(got, want, tol, "out")
        _check(lse, want_lse, tol_lse, "lse")


def _slopes(Hq):
    return torch.exp2(-8.0 * torch.arange(1, Hq + 1).float() / Hq)


DENSE = [("f32", 1, 1, 1, 1, 1), ("bf16", 1, 1, 4, 1, 1), ("bf16", 2, 5, 8, 2, 33), ("f32", 2, 5, 8, 2, 100), ("fp8", 1, 3, 4, 1, 64),
         ("bf16", 1, 64, 8, 1, 200), ("bf16", 3, 33, 2, 2, 511), ("f32", 1, 40, 4, 2, 257), ("fp8", 2, 16, 8, 2, 700), ("bf16", 1, 1, 8, 1, 3001),
         ("bf16", 9, 2, 4, 4, 31), ("fp8", 1, 64, 8, 1, 95)]


@pytest.mark.parametrize("dtype,S,T,Hq,Hkv,N", DENSE)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_dense(dtype, S, T, Hq, Hkv, N, out):
    Case(dtype, S, T, Hq, Hkv, N, ragged=S > 1, seed=N).cache().compare(out)


LISTS = [("bf16", 1, 1, 4, 1, 600, 16, 3, "shared"), ("f32", 2, 4, 2, 2, 333, 16, 4, "own"), ("bf16", 2, 16, 8, 2, 900, 32, 5, "own"),
         ("fp8", 1, 8, 4, 1, 700, 32, 6, "own"), ("fp8", 3, 3, 8, 4, 200, 16, 16, "shared"), ("bf16", 1, 64, 4, 1, 2500, 64, 7, "own"),
         ("bf16", 1, 40, 8, 1, 3000, 1024, 60, "own"), ("f32", 1, 64, 1, 1, 1500, 512, 40, "own"), ("bf16", 2, 7, 4, 2, 50, 64, 9, "own"),
         ("bf16", 1, 5, 4, 1, 400, 16, 0, "shared"), ("bf16", 1, 2, 2, 1, 20000, 8192, 300, "shared")]


@pytest.mark.parametrize("dtype,S,T,Hq,Hkv,N,B,nprobe,lists", LISTS)
@pytest.mark.parametrize("window", [None, (1, 47), (3, 0)])
def test_lists(dtype, S, T, Hq, Hkv, N, B, nprobe, lists, window):
    Case(dtype, S, T, Hq, Hkv, N, B, nprobe, lists, window, seed=B).cache().compare(torch.float32 if N % 2 else torch.bfloat16)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("what", ["cap", "bias", "starts", "all", "cap without drafts", "nothing seen"])
@pytest.mark.parametrize("lists", ["none", "own"])
def test_shaped_scores(dtype, what, lists):
    c = Case(dtype, 2, 6, 8, 2, 700, 32, 6, lists, (1, 30) if lists == "own" else None, seed=3).cache()
    cap = 3.0 if what in ("cap", "all", "cap without drafts") else 0.0
    slopes = _slopes(8) if what in ("bias", "all") else None
    starts = None
    if what in ("starts", "all"):
        starts = torch.randint(0, 900, (2, 6), generator=c.g).to(torch.int32)
        starts[0, 0], starts[1, 1] = 0, 699
    if what == "nothing seen":
        starts = torch.full((2, 6), 700, dtype=torch.int32)
        c.tree[1, 2] = 0
        c.compare(starts=starts, drafts=False)
    c.compare(softcap=cap, slopes=slopes, starts=starts, drafts=what != "cap without drafts")


def test_far_keys_and_steep_slopes_lose_nothing():
    """Keys 200000 positions back with slopes of 1/2: scores of -10^5, of which only differences count."""
    c = Case("f32", 1, 3, 4, 1, 500, seed=5).cache()
    c.pos = c.pos + 200000
    c.compare(slopes=torch.tensor([0.5, 0.25, 0.01, -0.03]), drafts=False)


def test_the_largest_row_count_and_long_lists():
    Case("bf16", 1, 64, 8, 1, 5000, 256, 200, "own", (4, 100), seed=6).cache().compare()


def test_what_is_masked_does_not_matter():
    """Infinities and NaN in drafted tokens that nobody attends, behind a sequence's keys, in other buckets, in free slots and
    before the starts; then in keys that some rows attend: those rows alone are no numbers."""
    nan, inf = float("nan"), float("inf")
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 2, 6, 4, 2, 300, ragged=True, seed=8).cache()
        c.n_keys = torch.tensor([120, 300], dtype=torch.int32)
        c.seen = (c.kpos < c.n_keys[:, None, None, None]).expand(2, 2, 6, -1)
        c.tree = saap.tree_masks(torch.tensor([[-1, 0, 0, 1, 6, 6], [-1, -1, 1, 6, 6, 6]]))
        want, want_lse = c.run()
        c.Kd[0, :, 120:] = nan
        c.Vd[0, :, 120:] = inf
        for s, n in ((0, 4), (1, 3)):
            c.kt[s, :, n:], c.vt[s, :, n:] = -inf, nan
        got, lse = c.run()
        assert torch.equal(got, want) and torch.equal(lse, want_lse)
        # one drafted value that tokens 1 and 3 of the first tree attend
        c.vt[0, 1, 1, 7] = inf
        got, lse = c.run()
        mine = torch.zeros(2, 6, 4, dtype=torch.bool)
        mine[0, 1, 2:] = mine[0, 3, 2:] = True
        assert torch.equal(lse, want_lse)
        assert (got[..., 7].cpu()[mine] == inf).all() and torch.equal(got[..., 7].cpu()[~mine], want[..., 7].cpu()[~mine])
        rest = [f for f in range(128) if f != 7]
        assert torch.allclose(got[..., rest], want[..., rest], rtol=1e-5, atol=1e-5)
        # a key that is no number makes its rows no numbers
        c.kt[0, 1, 1, 0] = nan
        got, _ = c.run()
        assert got.cpu()[mine].isnan().all() and torch.equal(got.cpu()[~mine], want.cpu()[~mine])


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
def test_values_of_other_lists(dtype):
    c = Case(dtype, 1, 5, 4, 1, 600, 16, 4, "own", seed=9).cache(slack=5)
    want, want_lse = c.run()
    unlisted = sorted(set(range(16)) - set(c.sel[0, :, 0].flatten().tolist()))
    only_0 = sorted(set(c.sel[0, 0, 0].tolist()) - set(c.sel[0, 1:, 0].flatten().tolist()))
    off, ln = c.off[0, 0].tolist(), c.ln[0, 0].tolist()
    no = 0x7f if dtype == "fp8" else float("nan")
    for b in range(16):
        c.Kd[0, 0, off[b] + ln[b]:off[b + 1]] = no           # free slots
        c.Vd[0, 0, off[b] + ln[b]:off[b + 1]] = no
    for b in unlisted:
        c.Kd[0, 0, off[b]:off[b + 1]] = no
        c.Vd[0, 0, off[b]:off[b + 1]] = no
    got, lse = c.run()
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    if only_0:
        c.Vd[0, 0, off[only_0[0]], 3] = no
        got, _ = c.run()
        assert got[0, 0, :, 3].isnan().all() and torch.equal(got[0, 1:, :, 3], want[0, 1:, :, 3])
        assert torch.allclose(got[..., 4:], want[..., 4:], rtol=1e-5, atol=1e-5)


def test_a_token_alone_has_the_result_that_it_has_in_the_tree():
    """Own lists: every drafted token is decoded as if it stood alone behind its ancestors."""
    c = Case("bf16", 2, 9, 8, 2, 1200, 32, 4, "own", (1, 63), seed=10).cache()
    whole, whole_lse = c.run()
    for t in (0, 4, 8):
        d = lambda x: x.to(DEV)  # noqa: E731
        one = torch.zeros_like(c.tree)
        one[:, t] = c.tree[:, t]
        got, lse = saap.tree_decode_attention(d(c.q), c.Kd, c.Vd, c.off, c.ln, d(c.sel[:, t].contiguous()), SCALE, d(c.kt), d(c.vt), d(one),
                                              resident_run=32)
        assert torch.allclose(got[:, t], whole[:, t], rtol=1e-4, atol=2e-5) and torch.allclose(lse[:, t], whole_lse[:, t], rtol=1e-5, atol=1e-5)


def test_equal_to_the_single_token_calls():
    c = Case("bf16", 2, 1, 8, 2, 2000, 32, 5, "shared", seed=12).cache()
    got, lse = c.run(drafts=False)
    want, want_lse = saap.sparse_decode_attention(c.q[:, 0].to(DEV), c.Kd, c.Vd, c.off, c.ln, c.sel.to(DEV), SCALE)
    assert torch.allclose(got[:, 0], want, rtol=1e-4, atol=2e-5) and torch.allclose(lse[:, 0], want_lse, rtol=1e-5, atol=1e-5)


def test_ids_out_of_range_and_twice():
    c = Case("bf16", 1, 4, 4, 1, 500, 16, 5, "own", seed=13).cache()
    want, want_lse = c.run()
    sel = c.sel
    odd = torch.tensor([-1, 16, 99, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).expand(1, 4, 1, 5)
    c.sel = torch.cat((sel[..., 2:], odd, sel, sel[..., :1]), -1)[..., :16].contiguous()
    got, lse = c.run()
    assert torch.equal(got, want) and torch.equal(lse, want_lse)


def test_captured_and_on_two_streams():
    c = Case("bf16", 2, 9, 8, 2, 1500, 32, 6, "own", (1, 31), seed=14).cache()
    d = Case("bf16", 1, 40, 8, 1, 900, seed=15).cache()
    args = dict(q=c.q.to(DEV), Ks=c.Kd, Vs=c.Vd, off=c.off, ln=c.ln, selected=c.sel.to(DEV), scale=SCALE, k_tree=c.kt.to(DEV),
                v_tree=c.vt.to(DEV), tree=c.tree.to(DEV), resident_run=32)
    dense = (d.q.to(DEV), d.Kd, d.Vd, SCALE, d.kt.to(DEV), d.vt.to(DEV), d.tree.to(DEV))
    both = lambda: saap.tree_decode_attention(**args) + saap.dense_tree_decode_attention(*dense)  # noqa: E731
    want = both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        eager = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, e) for a, b, e in zip(out, want, eager))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = both()
    here = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, e) for a, b, e in zip(want, here, there))


def test_outputs_passed_in():
    c = Case("bf16", 1, 4, 4, 1, 100, seed=16).cache()
    out, lse = torch.empty(1, 4, 4, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 4, 4, device=DEV)
    got = c.run(out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    want, want_lse = c.run(torch.bfloat16)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
