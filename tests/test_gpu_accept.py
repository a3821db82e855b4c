"""append_accepted: the index that append_keys or window_push, called for one token after the other, leaves; and a run of the
calls for drafted tokens together."""
import math

import pytest
import torch

import paper_2502_08246_amd as saap

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _index(S, Hkv, N, B, slack, dtype, window, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)  # noqa: E731
    cent = rand(Hkv, B, 128)
    K, V = rand(S, Hkv, N, 128), rand(S, Hkv, N, 128)
    ids = saap.assign_keys(K, cent)
    if window:
        index = list(saap.build_windowed_index(ids, K, V, B, slack, *window))
    else:
        index = list(saap.build_bucket_index(ids, K, V, B, slack)) + [None]
    return g, rand, cent, index


def _one_by_one(index, cent, x, k, v, path, pos_new, window, scales=()):
    """The calls for single tokens; a sequence whose path has ended is taken out of the call."""
    off, ln, idx, Ks, Vs, res = index
    flag = torch.zeros(4, dtype=torch.int32, device=DEV)
    for i in range(path.shape[1]):
        for s in range(path.shape[0]):
            if (path[s, :i + 1] < 0).any() or (path[s, :i + 1] >= k.shape[2]).any():
                continue
            t, one = int(path[s, i]), slice(s, s + 1)
            row = lambda z: z[one, :, t].contiguous()  # noqa: E731
            pos = None if pos_new is None else (pos_new[one] + i).to(torch.int32)
            head = (row(x), row(k), row(v), pos, cent, None, off[one], ln[one], idx[one], Ks[one], Vs[one]) + tuple(z[one] for z in scales)
            if window:
                push = saap.window_push_fp8 if scales else saap.window_push
                ring = res[one] if res.numel() else torch.zeros(1, 1, 1, dtype=torch.int32, device=DEV)   # it wants an address
                push(*head, ring, *window, overflow_flag=flag)
            else:
                append = saap.append_keys_fp8 if scales else saap.append_keys
                append(*head, overflow_flag=flag)
    return flag


CASES = [  # S, Hkv, N, B, slack, T, P, window
    (1, 1, 300, 16, 8, 1, 1, None), (3, 2, 500, 16, 32, 12, 9, None), (2, 4, 700, 32, 1, 33, 20, None), (2, 1, 200, 16, 0, 5, 3, None),
    (2, 1, 300, 16, 80, 64, 64, None), (1, 2, 300, 16, 8, 9, 5, (1, 31)), (3, 2, 500, 16, 40, 24, 12, (2, 60)),
    (2, 2, 400, 16, 1, 24, 20, (0, 20)), (2, 2, 10, 16, 30, 24, 9, (4, 16)), (1, 2, 100, 16, 30, 9, 4, (6, 0)), (1, 2, 3, 16, 30, 9, 8, (6, 0)),
    (1, 2, 100, 16, 30, 9, 4, (0, 0)),
]


@pytest.mark.parametrize("S,Hkv,N,B,slack,T,P,window", CASES)
@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
def test_as_one_by_one(S, Hkv, N, B, slack, T, P, window, kind):
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    g, rand, cent, index = _index(S, Hkv, N, B, slack, dtype, window, seed=N + T)
    x, k, v = rand(S, Hkv, T, 128), rand(S, Hkv, T, 128), rand(S, Hkv, T, 128)
    path = torch.randint(0, T, (S, P), generator=g, device=DEV).to(torch.int32)      # a token may come twice
    if S > 1:
        path[0, P // 2:] = -1
        path[1, P - 1] = T
    pos_new = torch.full((S,), N, dtype=torch.int32, device=DEV)
    scales = ()
    if kind == "fp8":
        index[3], index[4], *scales = saap.quantize_kv(index[3], index[4])
    theirs = [None if t is None else t.clone() for t in index]
    want_flag = _one_by_one(theirs, cent, x, k, v, path, pos_new, window, tuple(scales))
    ids = saap.assign_keys(x, cent)
    off, ln, idx, Ks, Vs, res = index
    more = {} if window is None else dict(resident_ids=res, n_sink=window[0], n_recent=window[1])
    call = saap.append_accepted_fp8 if scales else saap.append_accepted
    flag = call(ids, k, v, path, pos_new, off, ln, idx, Ks, Vs, *scales, **more)
    assert int(flag[0]) == int(want_flag[0])
    for name, a, b in zip(("off", "len", "idx", "Ks", "Vs", "resident_ids"), index, theirs):
        assert a is None or torch.equal(a, b), name


def test_no_positions_and_nothing_accepted():
    g, rand, cent, index = _index(2, 2, 200, 16, 10, torch.bfloat16, None, seed=3)
    before = [t.clone() for t in index[:5]]
    x, k = rand(2, 2, 6, 128), rand(2, 2, 6, 128)
    ids = saap.assign_keys(x, cent)
    none = torch.full((2, 4), -1, dtype=torch.int32, device=DEV)
    flag = saap.append_accepted(ids, k, k, none, None, *index[:5])
    assert int(flag.sum()) == 0 and all(torch.equal(a, b) for a, b in zip(index, before))
    path = torch.tensor([[0, 3, 5, -1], [1, 2, -1, 4]], dtype=torch.int32, device=DEV)
    theirs = [t.clone() for t in before] + [None]
    _one_by_one(theirs, cent, x, k, k, path, None, None)
    saap.append_accepted(ids, k, k, path, None, *index[:5], overflow_flag=flag)
    assert int(flag.sum()) == 0 and all(torch.equal(a, b) for a, b in zip(index[:5], theirs))


def test_ids_outside_the_buckets_are_refused_and_others_stored():
    g, rand, cent, index = _index(1, 1, 100, 16, 10, torch.bfloat16, None, seed=4)
    k = rand(1, 1, 4, 128)
    ids = torch.tensor([[[2, 16, -1, 2]]], dtype=torch.int32, device=DEV)
    path = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    before = index[1].clone()
    flag = saap.append_accepted(ids, k, k, path, torch.tensor([100], dtype=torch.int32, device=DEV), *index[:5])
    before[0, 0, 2] += 2
    assert int(flag[0]) == 1 and torch.equal(index[1], before)
    at = int(index[0][0, 0, 2] + index[1][0, 0, 2])
    assert index[2][0, 0, at - 2:at].tolist() == [100, 103]
    assert torch.equal(index[3][0, 0, at - 2:at], k[0, 0, [0, 3]])


def test_captured():
    g, rand, cent, index = _index(2, 2, 200, 16, 40, torch.bfloat16, None, seed=5)
    x, k = rand(2, 2, 6, 128), rand(2, 2, 6, 128)
    ids = saap.assign_keys(x, cent)
    path = torch.tensor([[0, 3, 5, -1], [1, 2, 4, 5]], dtype=torch.int32, device=DEV)
    pos = torch.full((2,), 200, dtype=torch.int32, device=DEV)
    flag = torch.zeros(4, dtype=torch.int32, device=DEV)
    theirs = [t.clone() for t in index[:5]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        saap.append_accepted(ids, k, k, path, pos, *index[:5], overflow_flag=flag)
    for _ in range(3):
        graph.replay()
        saap.append_accepted(ids, k, k, path, pos, *theirs)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(index, theirs))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_a_step_with_drafted_tokens(kind):
    """Projection -> norm and rotation -> routing of every drafted token -> attention of the tree -> the accepted branch joins the
    cache -> the next step's single token sees it.  Against the same steps on position-ordered tensors in 64 bits."""
    S, T, Hq, Hkv, N, B, nprobe, window = 2, 7, 8, 2, 600, 16, 5, (1, 63)
    g = torch.Generator(device=DEV).manual_seed(21)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    bf = torch.bfloat16
    freqs = saap.rotary_frequencies(64, scaling="bands", factor=4.0, context=512)
    qw, kw = 1 + 0.2 * rand(128), 1 + 0.2 * rand(128)
    cent = rand(Hkv, B, 128).to(bf)
    heads = Hq + 2 * Hkv
    scale = 1 / math.sqrt(128)

    def project(tokens):
        rows = rand(S, tokens, heads * 128).to(bf)
        split = lambda a, b: rows[..., a * 128:b * 128].unflatten(2, (b - a, 128))  # noqa: E731
        return split(0, Hq), split(Hq, Hq + Hkv), split(Hq + Hkv, heads).transpose(1, 2).contiguous()

    # the prompt
    q, k, v = project(N)
    at = torch.arange(N, device=DEV, dtype=torch.int32).expand(S, N).contiguous()
    _, _, k_rot, k_feat = saap.norm_rotate(None, k, at, freqs, k_weight=kw, pairs=True)
    ids = saap.assign_keys(k_feat, cent)
    off, ln, idx, Ks, Vs, res = saap.build_windowed_index(ids, k_rot, v, B, 20, *window)
    cache = (Ks, Vs)
    if kind == "fp8":
        K8, V8, ks, vs = saap.quantize_kv(Ks, Vs)
        cache = (K8, V8, ks, vs)

    # a tree of drafted tokens
    parents = torch.tensor([[-1, 0, 0, 1, 1, 4, 5], [-1, 0, 1, 2, 7, 7, 7]])
    tree = saap.tree_masks(parents).to(DEV)
    depth = torch.tensor([[0, 1, 1, 2, 2, 3, 4], [0, 1, 2, 3, 0, 0, 0]])
    pos = (N + depth).to(torch.int32).to(DEV)
    q, kt, vt = project(T)
    q_rot, q_feat, kt_rot, kt_feat = saap.norm_rotate(q, kt, pos, freqs, qw, kw, pairs=True)
    scores = saap.classify_queries(q_feat.view(S * T, Hq, 128), None, None, cent, None, Hkv)
    sel = saap.select_buckets(scores, Hkv, nprobe).view(S, T, Hkv, nprobe)
    attend = saap.tree_decode_attention_fp8 if kind == "fp8" else saap.tree_decode_attention
    out, _ = attend(q_rot, *cache, off, ln, sel, scale, kt_rot, vt, tree, resident_run=B)

    def held(x, unit_scale):
        if kind != "fp8":
            return x.double()
        return (x.float() / unit_scale[:, :, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).double() * unit_scale[:, :, None, None].double()

    K = held(k_rot, cache[2] if kind == "fp8" else None)
    V = held(v, cache[3] if kind == "fp8" else None)
    G = Hq // Hkv

    def wanted(s, t, hq, qr, lists, K, V, ids, n, drafts):
        h = hq // G
        p = torch.arange(n, device=DEV)
        see = (p < window[0]) | (p >= N - window[1]) if drafts else (p < window[0]) | (p >= n - window[1])
        see = see | torch.isin(ids[s, h], lists[s, t, h])
        kk, vv = K[s, h][see], V[s, h][see]
        if drafts:
            mine = ((tree[s, t] >> torch.arange(T, device=DEV)) & 1).bool()
            kk, vv = torch.cat((kk, kt_rot[s, h][mine].double())), torch.cat((vv, vt[s, h][mine].double()))
        return torch.softmax(kk @ qr[s, t, hq].double() * scale, 0) @ vv

    for s, t, hq in [(0, 0, 0), (0, 6, 5), (1, 3, 7), (0, 4, 2), (1, 0, 3)]:
        want = wanted(s, t, hq, q_rot, sel, K, V, ids, N, True)
        assert torch.allclose(out[s, t, hq].double(), want, rtol=1e-4, atol=1e-4), (s, t, hq)

    # 4 tokens of the first tree and 2 of the second are kept
    path = torch.tensor([[0, 1, 4, 5, -1], [0, 1, -1, -1, -1]], dtype=torch.int32, device=DEV)
    pos_new = torch.full((S,), N, dtype=torch.int32, device=DEV)
    t_ids = saap.assign_keys(kt_feat, cent)
    accept = saap.append_accepted_fp8 if kind == "fp8" else saap.append_accepted
    flag = accept(t_ids, kt_rot, vt, path, pos_new, off, ln, idx, *cache, resident_ids=res, n_sink=window[0], n_recent=window[1])
    assert int(flag[0]) == 0

    # the next token of either sequence, alone; its key is attended as a tree of one
    q, k1, v1 = project(1)
    now = torch.tensor([[N + 4], [N + 2]], dtype=torch.int32, device=DEV)
    q_rot, q_feat, k1_rot, _ = saap.norm_rotate(q, k1, now, freqs, qw, kw, pairs=True)
    sel = saap.select_buckets(saap.classify_queries(q_feat[:, 0].contiguous(), None, None, cent, None, Hkv), Hkv, nprobe)
    out, _ = attend(q_rot, *cache, off, ln, sel, scale, resident_run=B)
    for s, n in ((0, 4), (1, 2)):
        kept = path[s, :n].long()
        K1 = torch.cat((K[s:s + 1], held(kt_rot[s:s + 1, :, kept], cache[2][s:s + 1] if kind == "fp8" else None)), 2)
        V1 = torch.cat((V[s:s + 1], held(vt[s:s + 1, :, kept], cache[3][s:s + 1] if kind == "fp8" else None)), 2)
        all_ids = torch.cat((ids[s:s + 1], t_ids[s:s + 1, :, kept]), 2)
        for hq in (0, 5):
            want = wanted(0, 0, hq, q_rot[s:s + 1], sel[s:s + 1, None], K1, V1, all_ids, N + n, False)
            assert torch.allclose(out[s, 0, hq].double(), want, rtol=1e-4, atol=1e-4), (s, hq)
