"""The operators around a bucketed cache that drafted tokens need, as cases that can be timed and compared.

Four of them, in the order in which a program with drafted tokens calls them: the norm of every head's queries and keys with
the rotation by their positions ("rotate"), its gradients ("grads"), attention of a tree of drafted tokens over the cache
("tree", a single token being the smallest tree) and the storing of the accepted ones ("accept").  Where `own` is false they
are computed from elementary torch operations; where it is true the library is called.

Keys are N(0,1) per feature plus one offset per head, queries and values N(0,1), buckets of unequal sizes; the tokens of a tree
list the same buckets for half of their lists and buckets of their own for the rest.
"""
import math

import torch

own = False

D = 128                       # features per head
DEV = "cuda:0"
SCALE = 1.0 / math.sqrt(D)
THETA = 500000.0
N_SINK, N_RECENT = 1, 2047    # the dense window of the library's default setting
EPS = 1e-6
SIZE = {"f32": 4, "bf16": 2, "fp8": 1}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rotate(name, **kw):
    case = dict(name=name, path="rotate", S=1, T=1, Hq=32, Hkv=8, rot=128, layout="half", scaling="none", norm=True,
                per_head=False, fused=True, q_features=True, far=0, dtype="bf16")
    case.update(kw)
    return case


def _tree(name, **kw):
    case = dict(name=name, path="tree", S=1, T=1, Hq=32, Hkv=8, N=131072, B=1024, nprobe=51, lists="own", window=False,
                softcap=0.0, slopes=False, starts=False, ragged=False, out="f32", dtype="bf16")
    case.update(kw)
    return case


def _accept(name, **kw):
    case = dict(name=name, path="accept", S=1, T=16, P=8, Hkv=8, N=16384, B=128, dtype="bf16")
    case.update(kw)
    return case


def listed():
    return [
        # the smallest call: one decode step's queries and keys of a layer; latency is all there is
        _rotate("rotate_one_token"),
        # a prompt's queries and keys, read out of the fused projection; the keys' features are kept for their buckets
        _rotate("rotate_prompt_128k", T=131072, q_features=False, scaling="bands"),
        # an odd batch in fp32, neighbouring pairs, half of the head turned, weights per head
        _rotate("rotate_ragged_f32", S=3, T=1237, Hq=16, Hkv=4, rot=64, layout="pairs", per_head=True, fused=False, dtype="f32"),
        # a training batch: gradients of the inputs and of the shared weights
        _rotate("grads_batch4_4k", path="grads", S=4, T=4096),
        # the same for an odd length in fp32 with weights per head
        _rotate("grads_ragged_f32", path="grads", T=777, Hq=16, Hkv=16, rot=96, layout="pairs", per_head=True, fused=False,
                dtype="f32"),
        # single-token decoding of a model with capped scores over its listed buckets
        _tree("tree_one_token_capped", lists="shared", softcap=30.0),
        # a tree of 16 drafted tokens, each with its own list, sink and recent keys always attended
        _tree("tree_16_own_lists_window", T=16, window=True),
        # batched decoding with small trees on an 8-bit cache, one list per group
        _tree("tree_batch8_fp8", S=8, T=8, lists="shared", dtype="fp8", out="bf16"),
        # the largest: 64 drafted tokens over every key of a long context
        _tree("tree_64_dense_128k", T=64, lists="none", out="bf16"),
        # a short fp32 cache, sequences of unequal lengths, distance bias and documents that begin inside the cache
        _tree("tree_ragged_dense_f32", S=5, T=5, Hq=4, Hkv=1, N=4096, lists="none", slopes=True, starts=True, ragged=True,
              dtype="f32"),
        # what a batch of trees keeps: up to 8 of 16 drafted tokens each
        _accept("accept_batch8", S=8),
        # one short fp32 sequence
        _accept("accept_one_f32", T=5, P=3, Hkv=1, N=4096, B=64, dtype="f32"),
    ]


# ------------------------------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return rng.choice([(32, 8), (32, 8), (64, 8), (16, 8), (8, 8), (4, 1), (16, 4), (2, 1), (1, 1)])


def _draw_rotate(rng, path):
    Hq, Hkv = _heads(rng)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    tokens = 131072 * 40 // (Hq + Hkv) // (2 if dtype == "f32" else 1) // (4 if path == "grads" else 2)
    S = _log_int(rng, 1, 32)
    return dict(path=path, S=S, T=_log_int(rng, 1, max(2, min(65536, tokens // S))), Hq=Hq, Hkv=Hkv,
                rot=rng.choice([128, 128, 128, 96, 64, 32]), layout=rng.choice(["half", "half", "pairs"]),
                scaling=rng.choice(["none", "linear", "base", "bands"]), norm=rng.random() < 0.8,
                per_head=rng.random() < 0.3, fused=rng.random() < 0.6, q_features=rng.random() < 0.5,
                far=rng.choice([0, 0, 100000, 10000000]), dtype=dtype)


def _draw_tree(rng):
    Hq, Hkv = _heads(rng)
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp8", "fp8", "f32"])
    lists = rng.choice(["own", "own", "shared", "none"])
    N = _log_int(rng, 700, 16384 if dtype == "f32" else 131072)
    T = min(64, _log_int(rng, 1, 64))
    most = 131072 * 8 * 256 // (N * Hkv * max(32, T * Hq // Hkv)) // (4 if dtype == "f32" else 2)
    S = max(1, min(_log_int(rng, 1, 32), most))
    if most < 1:
        T = max(1, T // 4)
    B = max(16, min(2048, 16 * int(round(N / math.exp(rng.uniform(math.log(32), math.log(256))) / 16))))
    return dict(path="tree", S=S, T=T, Hq=Hq, Hkv=Hkv, N=N, B=B,
                nprobe=max(1, int(round(B * math.exp(rng.uniform(math.log(0.01), math.log(0.12)))))), lists=lists,
                window=lists != "none" and N > 4 * N_RECENT and rng.random() < 0.4,
                softcap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.3, starts=rng.random() < 0.3,
                ragged=lists == "none" and rng.random() < 0.5, out=rng.choice(["f32", "bf16"]), dtype=dtype)


def _draw_accept(rng):
    N = _log_int(rng, 700, 16384)
    T = _log_int(rng, 1, 64)
    return dict(path="accept", S=_log_int(rng, 1, 16), T=T, P=rng.randint(1, min(T, 24)), Hkv=rng.choice([8, 8, 4, 1]), N=N,
                B=max(16, 16 * (N // 2048)), dtype=rng.choice(["bf16", "bf16", "f32"]))


def draw(rng):
    path = rng.choice(["rotate", "rotate", "grads", "tree", "tree", "tree", "accept"])
    if path == "tree":
        return _draw_tree(rng)
    return _draw_accept(rng) if path == "accept" else _draw_rotate(rng, path)


# ------------------------------------------------------------------------------------------ inputs
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _frequencies(rot, scaling):
    """Radians per position of every pair, in double precision: theta^(-2i/rot), then scaled for a context 8 times as long as
    the 8192 positions of training.  linear: all of them slower; base: a larger theta; bands: slow ones slower, fast ones as
    they are, a blend between (1 to 4 turns over the trained context)."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    factor, trained = 8.0, 8192.0
    theta = THETA * factor ** (rot / (rot - 2)) if scaling == "base" else THETA
    f = theta ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":
        keep = ((trained * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = keep * f + (1 - keep) * f / factor
    return f


def _prepare_rotate(case, gen):
    S, T, Hq, Hkv, dtype = case["S"], case["T"], case["Hq"], case["Hkv"], TORCH[case["dtype"]]
    st = {}
    if case["fused"]:         # queries, keys and values of a token side by side, as one projection writes them
        rows = _randn(gen, S, T, (Hq + 2 * Hkv) * D).to(dtype)
        st["q"] = rows[:, :, :Hq * D].unflatten(2, (Hq, D))
        st["k"] = rows[:, :, Hq * D:(Hq + Hkv) * D].unflatten(2, (Hkv, D))
    else:
        st["q"], st["k"] = _randn(gen, S, T, Hq, D).to(dtype), _randn(gen, S, T, Hkv, D).to(dtype)
    first = torch.randint(0, 4096, (S, 1), generator=gen, device=DEV) + case["far"]
    st["positions"] = (first + torch.arange(T, device=DEV)).to(torch.int32)
    st["freqs"] = _frequencies(case["rot"], case["scaling"]).to(DEV)
    st["magnitude"] = 1.0 if case["scaling"] in ("none", "linear") else 1.0 + 0.1 * math.log(8.0)
    for n, H in (("q_weight", Hq), ("k_weight", Hkv)):
        st[n] = 1.0 + 0.2 * _randn(gen, *((H, D) if case["per_head"] else (D,))) if case["norm"] else None
    if case["path"] == "grads":
        st["g_q_feat"] = _randn(gen, S, T, Hq, D).to(dtype) if case["q_features"] else None
        st["g_q_rot"] = _randn(gen, S, T, Hq, D).to(dtype)
        st["g_k_feat"], st["g_k_rot"] = _randn(gen, S, Hkv, T, D).to(dtype), _randn(gen, S, Hkv, T, D).to(dtype)
    return st


def _index(gen, S, Hkv, N, B, slack, window):
    """off, len, idx and the slots' number of an index over N keys with unequal buckets, as a build writes them."""
    W = N_SINK + N_RECENT if window else 0
    units, runs = S * Hkv, B + (1 if window else 0)
    share = torch.exp(0.5 * _randn(gen, units, B))
    bucket = torch.multinomial(share, N, replacement=True, generator=gen)
    where = torch.arange(N, device=DEV).expand(units, N)
    if window:                # sink and recent keys are in the run behind the buckets
        bucket = torch.where((where < N_SINK) | (where >= N - N_RECENT), B, bucket)
    length = torch.zeros(units, runs, dtype=torch.int64, device=DEV).scatter_add_(1, bucket, torch.ones_like(bucket))
    room = length + slack
    if window:
        room[:, B] = W
    off = torch.zeros(units, runs + 1, dtype=torch.int64, device=DEV)
    off[:, 1:] = room.cumsum(1)
    Ncap = N + B * slack
    order = torch.sort(bucket, dim=1, stable=True).indices
    run = bucket.gather(1, order)
    rank = where - (length.cumsum(1) - length).gather(1, run)
    if window:                # the recent part is a ring
        r = torch.where(order < N_SINK, order, N_SINK + (order - N_SINK) % N_RECENT)
        rank = torch.where(run == B, r, rank)
    idx = torch.full((units, Ncap), -1, dtype=torch.int64, device=DEV).scatter_(1, off.gather(1, run) + rank, order)
    shape = lambda t: t.to(torch.int32).view(S, Hkv, -1).contiguous()  # noqa: E731
    return shape(off), shape(length), shape(idx), Ncap


def _drafts(gen, S, T, ragged_from=None):
    """A random tree per sequence: which drafted tokens each of them sees (itself and its ancestors), as bits; a padded batch
    has trees of fewer tokens, whose last rows see nothing."""
    parent = (torch.rand(S, T, generator=gen, device=DEV) * torch.arange(T, device=DEV).clamp(min=1)).long()
    sees = torch.zeros(S, T, T, dtype=torch.bool, device=DEV)
    rows = torch.arange(S, device=DEV)
    depth = torch.zeros(S, T, dtype=torch.int64, device=DEV)
    for t in range(T):
        if t:
            sees[:, t] = sees[rows, parent[:, t]]
            depth[:, t] = depth[rows, parent[:, t]] + 1
        sees[:, t, t] = True
    if T > 2:
        count = torch.randint(T // 2 + 1, T + 1, (S,), generator=gen, device=DEV)
        sees &= (torch.arange(T, device=DEV) < count[:, None])[:, :, None]
    tree = (sees.long() << torch.arange(T, device=DEV)).sum(2)
    return tree, depth


def _cache(gen, S, Hkv, rows, dtype):
    offset = _randn(gen, Hkv, 1, D)
    K = (_randn(gen, S, Hkv, rows, D) + offset).to(dtype)
    return K, _randn(gen, S, Hkv, rows, D).to(dtype)


def _to_fp8(x):
    """Codes and one power-of-two scale per (sequence, head)."""
    top = x.float().abs().amax((2, 3))
    scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)))
    return (x.float() / scale[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _prepare_tree(case, gen):
    S, T, Hq, Hkv, N, B, nprobe = (case[k] for k in ("S", "T", "Hq", "Hkv", "N", "B", "nprobe"))
    fp8, dtype = case["dtype"] == "fp8", TORCH["bf16" if case["dtype"] == "fp8" else case["dtype"]]
    st = {"scale": SCALE, "softcap": case["softcap"], "out_dtype": TORCH[case["out"]], "kscale": None, "vscale": None}
    rows = N
    if case["lists"] != "none":
        st["off"], st["len"], st["idx"], rows = _index(gen, S, Hkv, N, B, 4, case["window"])
        st["resident_run"] = B if case["window"] else -1
        own_lists = case["lists"] == "own"
        # half of a list is the group's, the rest the token's own
        score = torch.rand(S, 1, Hkv, B, generator=gen, device=DEV) + torch.zeros(S, T if own_lists else 1, Hkv, 1, device=DEV)
        common = score[:, :1].topk((nprobe + 1) // 2, dim=3).indices
        score = torch.rand(score.shape, generator=gen, device=DEV).scatter(3, common.expand(-1, score.shape[1], -1, -1), 2.0)
        sel = score.topk(nprobe, dim=3).indices.to(torch.int32)
        st["selected"] = sel.contiguous() if own_lists else sel[:, 0].contiguous()
    else:
        st["selected"] = None
        st["n_keys"] = None
        if case["ragged"]:
            st["n_keys"] = torch.randint(0, N + 1, (S,), generator=gen, device=DEV).to(torch.int32)
            st["n_keys"][0] = N
    st["K"], st["V"] = _cache(gen, S, Hkv, rows, dtype)
    if fp8:
        st["K"], st["kscale"] = _to_fp8(st["K"])
        st["V"], st["vscale"] = _to_fp8(st["V"])
    st["q"] = (1.5 * _randn(gen, S, T, Hq, D)).to(dtype)
    st["tree"], depth = _drafts(gen, S, T)
    st["k_tree"], st["v_tree"] = _cache(gen, S, Hkv, T, dtype)
    st["slopes"] = st["pos"] = st["starts"] = None
    held = N if st.get("n_keys") is None else st["n_keys"].long()[:, None]
    if case["slopes"]:
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq)
        st["pos"] = (held + depth).to(torch.int32)
    if case["starts"]:
        st["starts"] = (torch.rand(S, 1, generator=gen, device=DEV) * (held + 1) * 0.9).to(torch.int32).expand(S, T).contiguous()
    return st


def _prepare_accept(case, gen):
    S, T, P, Hkv, N, B, dtype = case["S"], case["T"], case["P"], case["Hkv"], case["N"], case["B"], TORCH[case["dtype"]]
    st = {}
    st["off"], st["len"], st["idx"], Ncap = _index(gen, S, Hkv, N, B, 32, False)
    st["len_before"] = st["len"].clone()
    st["Ks"], st["Vs"] = _cache(gen, S, Hkv, Ncap, dtype)
    st["k_tree"], st["v_tree"] = _cache(gen, S, Hkv, T, dtype)
    st["ids"] = torch.randint(0, B, (S, Hkv, T), generator=gen, device=DEV).to(torch.int32)
    path = torch.rand(S, T, generator=gen, device=DEV).topk(P, dim=1).indices.sort(1).values
    count = torch.randint(1, P + 1, (S, 1), generator=gen, device=DEV)
    st["path"] = torch.where(torch.arange(P, device=DEV) < count, path, -1).to(torch.int32)
    st["pos_new"] = torch.full((S,), N, dtype=torch.int32, device=DEV)
    st["flag"] = torch.zeros(4, dtype=torch.int32, device=DEV)
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 7919 + 29)
    make = {"rotate": _prepare_rotate, "grads": _prepare_rotate, "tree": _prepare_tree, "accept": _prepare_accept}
    state = make[case["path"]](case, gen)
    state["case"] = case
    return state


# ------------------------------------------------------------------------------------------ one pass
def _turn(st, y, sign):
    """The first `rot` features of y [S,T,H,D] fp32 turned by sign * position * frequency."""
    rot, mag = 2 * st["freqs"].numel(), st["magnitude"]
    angle = st["positions"].double()[:, :, None] * st["freqs"]
    c, s = (mag * torch.cos(angle)).float()[:, :, None], (sign * mag * torch.sin(angle)).float()[:, :, None]
    if st["case"]["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        return torch.cat((a * c - b * s, b * c + a * s, y[..., rot:]), -1)
    a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    return torch.cat((torch.stack((a * c - b * s, b * c + a * s), -1).flatten(3), y[..., rot:]), -1)


def _plain_rotate(st):
    out = {}
    for n in ("q", "k"):
        y = st[n].float()
        if st["case"]["norm"]:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * st[n + "_weight"]
        rotated = _turn(st, y, 1.0)
        heads_first = (lambda t: t) if n == "q" else (lambda t: t.transpose(1, 2).contiguous())
        if n == "k" or st["case"]["q_features"]:
            out[n + "_feat"] = heads_first(y.to(st[n].dtype))
        out[n + "_rot"] = heads_first(rotated.to(st[n].dtype))
    return out


def _plain_grads(st):
    out = {}
    for n in ("q", "k"):
        x, w, g_feat, g_rot = st[n].float(), st[n + "_weight"], st[f"g_{n}_feat"], st[f"g_{n}_rot"].float()
        if n == "k":
            g_feat, g_rot = g_feat.transpose(1, 2), g_rot.transpose(1, 2)
        g = _turn_back(st, g_rot)
        if g_feat is not None:
            g = g + g_feat.float()
        if st["case"]["norm"]:
            r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
            u, xhat = g * w, x * r
            out["d" + n + "_weight"] = (g.double() * xhat).sum((0, 1) if w.dim() == 2 else (0, 1, 2)).float()
            g = r * (u - xhat * (u * xhat).mean(-1, keepdim=True))
        out["d" + n] = g.to(st[n].dtype)
    return out


def _turn_back(st, g):
    return _turn(st, g, -1.0)


def _decoded(st, name):
    x, scale = st[name], st["kscale" if name == "K" else "vscale"]
    return x.float() if scale is None else x.view(torch.float8_e4m3fn).float() * scale[:, :, None, None]


def _seen(st):
    """Which cached rows each token attends, [S,Hkv,T,rows] or [S,1,T,rows], and the rows' positions (the same shape or one that
    spreads to it)."""
    S, T = st["q"].shape[:2]
    rows = torch.arange(st["K"].shape[2], device=DEV)
    if st["selected"] is None:
        positions = rows[None, None, None]
        held = st["n_keys"]
        seen = torch.ones(S, 1, T, rows.numel(), dtype=torch.bool, device=DEV)
        if held is not None:
            seen &= rows < held[:, None, None, None]
    else:
        sel, off, ln = st["selected"].long(), st["off"].long(), st["len"].long()
        sel = sel[:, None] if sel.dim() == 3 else sel
        lists = torch.zeros(S, sel.shape[1], *ln.shape[1:], dtype=torch.bool, device=DEV).scatter_(3, sel, True)
        if st["resident_run"] >= 0:
            lists[..., st["resident_run"]] = True
        run = (torch.searchsorted(off, rows.expand(*off.shape[:2], -1).contiguous(), right=True) - 1).clamp(max=ln.shape[2] - 1)
        member = rows - off.gather(2, run) < ln.gather(2, run)
        lists = lists.transpose(1, 2).expand(-1, -1, T, -1)
        seen = lists.gather(3, run[:, :, None].expand(-1, -1, T, -1)) & member[:, :, None]
        positions = st["idx"].long()[:, :, None]
    if st["starts"] is not None:
        seen = seen & (positions >= st["starts"].long()[:, None, :, None])
    return seen, positions


def _plain_tree(st):
    q = st["q"].float()
    S, T, Hq, _ = q.shape
    Hkv = st["K"].shape[1]
    G = Hq // Hkv
    rows = q.view(S, T, Hkv, G, D).transpose(1, 2).reshape(S, Hkv, T * G, D)
    keys = torch.cat((_decoded(st, "K"), st["k_tree"].float()), 2)
    a = torch.matmul(rows, keys.transpose(2, 3)).view(S, Hkv, T, G, -1) * st["scale"]
    del keys
    if st["softcap"] > 0:
        a = st["softcap"] * torch.tanh(a / st["softcap"])
    seen, positions = _seen(st)
    if st["slopes"] is not None:        # products of far distances: in double precision
        at = torch.cat((positions.expand(S, Hkv, 1, -1), st["pos"].long()[:, None, None].expand(-1, Hkv, -1, -1)), 3)
        away = (st["pos"].long()[:, None, :, None] - at).double()
        a = a.double() - st["slopes"].double().view(1, Hkv, 1, G, 1) * away[:, :, :, None]
    drafted = ((st["tree"][:, :, None] >> torch.arange(T, device=DEV)) & 1).bool()[:, None].expand(-1, Hkv, -1, -1)
    seen = torch.cat((seen.expand(-1, Hkv, -1, -1), drafted), 3)[:, :, :, None]
    a = a.masked_fill(~seen, -math.inf)
    top = a.amax(-1, keepdim=True).clamp(min=-3.0e38)
    a = torch.exp(a - top)
    total = a.sum(-1, keepdim=True)
    values = torch.cat((_decoded(st, "V"), st["v_tree"].float()), 2)
    o = torch.matmul((a / total.clamp(min=1e-30)).float().reshape(S, Hkv, T * G, -1), values).view(S, Hkv, T, G, D)
    lse = (top + torch.log(total)).float().squeeze(-1)
    return {"out": o.transpose(1, 2).reshape(S, T, Hq, D).to(st["out_dtype"]), "lse": lse.transpose(1, 2).reshape(S, T, Hq)}


def _plain_accept(st):
    ids, path, off, ln = st["ids"].long(), st["path"].long(), st["off"].long(), st["len"]
    S, Hkv, T = ids.shape
    P = path.shape[1]
    live = (path >= 0).cumprod(1).bool()[:, None].expand(-1, Hkv, -1)
    node = path.clamp(min=0)[:, None].expand(-1, Hkv, -1)
    bucket = ids.gather(2, node)
    same = (bucket[:, :, :, None] == bucket[:, :, None]) & live[:, :, None]
    rank = (same & torch.ones(P, P, dtype=torch.bool, device=DEV).tril(-1)).sum(3)
    slot = off.gather(2, bucket) + ln.long().gather(2, bucket) + rank
    fits = slot < off.gather(2, bucket + 1)
    st["flag"][:1] |= (live & ~fits).any().to(torch.int32)
    put = live & fits
    s, h, i = put.nonzero(as_tuple=True)
    to = slot[s, h, i]
    st["Ks"][s, h, to] = st["k_tree"][s, h, node[s, h, i]]
    st["Vs"][s, h, to] = st["v_tree"][s, h, node[s, h, i]]
    st["idx"][s, h, to] = (st["pos_new"].long()[s] + i).to(torch.int32)
    ln.scatter_add_(2, bucket, put.to(torch.int32))


def run(st):
    case, path = st["case"], st["case"]["path"]
    if path == "accept":      # the lengths as they were before, so that every pass stores the same tokens
        st["len"].copy_(st["len_before"])
    if own:
        import paper_2502_08246_amd as saap
        if path == "rotate":
            got = saap.norm_rotate(st["q"], st["k"], st["positions"], st["freqs"], q_weight=st["q_weight"],
                                   k_weight=st["k_weight"], norm=case["norm"], eps=EPS, pairs=case["layout"] == "pairs",
                                   magnitude=st["magnitude"], q_features=case["q_features"])
            return {n: t for n, t in zip(("q_rot", "q_feat", "k_rot", "k_feat"), got) if t is not None}
        if path == "grads":
            got = saap.norm_rotate_grads(st["q"], st["k"], st["positions"], st["freqs"], st["g_q_rot"], st["g_q_feat"],
                                         st["g_k_rot"], st["g_k_feat"], q_weight=st["q_weight"], k_weight=st["k_weight"],
                                         norm=case["norm"], eps=EPS, pairs=case["layout"] == "pairs",
                                         magnitude=st["magnitude"])
            return {n: t for n, t in zip(("dq", "dk", "dq_weight", "dk_weight"), got) if t is not None}
        if path == "tree":
            scales = () if st["kscale"] is None else (st["kscale"], st["vscale"])
            more = dict(softcap=st["softcap"], slopes=st["slopes"], pos=st["pos"], starts=st["starts"],
                        out_dtype=st["out_dtype"])
            if st["selected"] is None:
                call = saap.dense_tree_decode_attention_fp8 if scales else saap.dense_tree_decode_attention
                out, lse = call(st["q"], st["K"], st["V"], *scales, st["scale"], st["k_tree"], st["v_tree"], st["tree"],
                                n_keys=st["n_keys"], **more)
            else:
                call = saap.tree_decode_attention_fp8 if scales else saap.tree_decode_attention
                out, lse = call(st["q"], st["K"], st["V"], *scales, st["off"], st["len"], st["selected"], st["scale"],
                                st["k_tree"], st["v_tree"], st["tree"], resident_run=st["resident_run"], idx=st["idx"], **more)
            return {"out": out, "lse": lse}
        saap.append_accepted(st["ids"], st["k_tree"], st["v_tree"], st["path"], st["pos_new"], st["off"], st["len"], st["idx"],
                             st["Ks"], st["Vs"], overflow_flag=st["flag"])
    elif path == "rotate":
        return _plain_rotate(st)
    elif path == "grads":
        return _plain_grads(st)
    elif path == "tree":
        return _plain_tree(st)
    else:
        _plain_accept(st)
    return {n: st[n] for n in ("len", "idx", "Ks", "Vs", "flag")}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def _rotation_matrix(st, s):
    """[T,D,D] fp64: what the rotation does to the features of sequence s's tokens."""
    rot = 2 * st["freqs"].numel()
    angle = st["positions"][s].double()[:, None] * st["freqs"]
    i = torch.arange(rot // 2, device=DEV)
    a, b = (i, i + rot // 2) if st["case"]["layout"] == "half" else (2 * i, 2 * i + 1)
    M = torch.eye(D, dtype=torch.float64, device=DEV).repeat(angle.shape[0], 1, 1)
    M[:, a, a] = M[:, b, b] = st["magnitude"] * torch.cos(angle)
    M[:, b, a] = st["magnitude"] * torch.sin(angle)
    M[:, a, b] = -M[:, b, a]
    return M


def _exact_rotate(st):
    case = st["case"]
    out, parts = {}, {}
    for n in ("q", "k"):
        for s in range(case["S"]):
            for t0 in range(0, case["T"], 8192):
                at = slice(t0, t0 + 8192)
                x = st[n][s, at].double()
                M = _rotation_matrix({**st, "positions": st["positions"][:, at]}, s)
                if case["norm"]:
                    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * st[n + "_weight"].double()
                parts.setdefault(n + "_feat", []).append(x)
                parts.setdefault(n + "_rot", []).append((M @ x.transpose(1, 2).contiguous()).transpose(1, 2))
    for name, got in parts.items():
        whole = torch.cat(got).view(case["S"], case["T"], -1, D)
        if name != "q_feat" or case["q_features"]:
            out[name] = whole if name[0] == "q" else whole.transpose(1, 2).contiguous()
    return out


def _exact_grads(st):
    """The derivative of sum(g_feat * features) + sum(g_rot * rotated), by the chain rule on whole matrices."""
    case, out = st["case"], {}
    for n in ("q", "k"):
        dx, dw = [], 0.0
        for s in range(case["S"]):
            for t0 in range(0, case["T"], 8192):
                at = slice(t0, t0 + 8192)
                x = st[n][s, at].double()
                M = _rotation_matrix({**st, "positions": st["positions"][:, at]}, s)
                mine = lambda g: (g[s, at] if n == "q" else g[s, :, at].transpose(0, 1)).double()  # noqa: E731
                g = mine(st[f"g_{n}_rot"]) @ M
                if st[f"g_{n}_feat"] is not None:
                    g = g + mine(st[f"g_{n}_feat"])
                if case["norm"]:
                    w = st[n + "_weight"].double()
                    size = torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS)
                    dw = dw + (g * x / size).sum((0,) if case["per_head"] else (0, 1))
                    g = g * w / size - x * ((g * w * x).sum(-1, keepdim=True) / (D * size ** 3))
                dx.append(g)
        out["d" + n] = torch.cat(dx).view(st[n].shape)
        if case["norm"]:
            out["d" + n + "_weight"] = dw
    return out


def _exact_tree(st):
    """One KV head at a time: scores, their logarithmic sum and the weighted values, over every row with a mask."""
    S, T, Hq, _ = st["q"].shape
    Hkv, rows = st["K"].shape[1:3]
    G = Hq // Hkv
    out = torch.zeros(S, T, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(S, T, Hq, dtype=torch.float64, device=DEV)
    drafted = torch.arange(T, device=DEV)
    for s in range(S):
        for h in range(Hkv):
            k, v = st["K"][s, h], st["V"][s, h]
            if st["kscale"] is not None:
                k, v = k.view(torch.float8_e4m3fn).float(), v.view(torch.float8_e4m3fn).float()
            k = k.double() * (1.0 if st["kscale"] is None else st["kscale"][s, h].double())
            v = v.double() * (1.0 if st["vscale"] is None else st["vscale"][s, h].double())
            if st["selected"] is None:
                where = torch.arange(rows, device=DEV)
                held = rows if st["n_keys"] is None else st["n_keys"][s].long()
                see = (where < held).expand(T, rows)
            else:
                where, room = st["idx"][s, h].long(), st["off"][s, h].long().diff()
                bucket = torch.repeat_interleave(torch.arange(room.numel(), device=DEV), room)
                bucket = torch.cat((bucket, torch.full((rows - bucket.numel(),), -1, device=DEV)))
                lists = st["selected"][s, h][None] if st["selected"].dim() == 3 else st["selected"][s, :, h]
                see = (bucket[None, :, None] == lists.long()[:, None]).any(2) if rows * lists.numel() < 1 << 28 else None
                if see is None:
                    see = torch.stack([torch.isin(bucket, one.long()) for one in lists])
                see = (see | (bucket == st["resident_run"]) & (bucket >= 0)) & (where >= 0)
                see = see.expand(T, rows)
            if st["starts"] is not None:
                see = see & (where >= st["starts"][s].long()[:, None])
            see = torch.cat((see, (st["tree"][s][:, None] >> drafted) % 2 == 1), 1)
            k, v = torch.cat((k, st["k_tree"][s, h].double())), torch.cat((v, st["v_tree"][s, h].double()))
            for g in range(G):
                a = st["q"][s, :, h * G + g].double() @ k.t().contiguous() * st["scale"]
                if st["softcap"] > 0:
                    a = st["softcap"] * torch.tanh(a / st["softcap"])
                if st["slopes"] is not None:
                    at = torch.cat((where, st["pos"][s].long()))
                    a = a - st["slopes"][h * G + g].double() * (st["pos"][s].long()[:, None] - at).double()
                a = torch.where(see, a, -math.inf)
                total = torch.logsumexp(a, 1)
                lse[s, :, h * G + g] = total
                out[s, :, h * G + g] = torch.exp(a - total.clamp(min=-1e300)[:, None]) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["path"] == "accept":        # moves rows, computes none
        return None
    st = prepare(case, seed)
    return {"rotate": _exact_rotate, "grads": _exact_grads, "tree": _exact_tree}[case["path"]](st)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e, S, T, Hkv = SIZE[case["dtype"]], case["S"], case["T"], case["Hkv"]
    if case["path"] == "accept":        # on average (P + 1) / 2 tokens: their K and V read and written
        return {"bytes": S * Hkv * (case["P"] + 1) // 2 * (4 * D * e + 16), "flops": 0}
    Hq = case["Hq"]
    q, k = S * T * Hq * D, S * T * Hkv * D
    feat = q if case.get("q_features") else 0
    if case["path"] == "rotate":
        return {"bytes": e * (2 * q + feat + 3 * k), "flops": 10 * (q + k)}
    if case["path"] == "grads":
        return {"bytes": e * (3 * q + feat + 4 * k), "flops": 16 * (q + k)}
    N, R = case["N"], T * Hq // Hkv
    union = mine = float(N) * (0.6 if case["ragged"] else 1.0)
    if case["lists"] != "none":
        common = (case["nprobe"] + 1) // 2
        rest, left = case["B"] - common, case["nprobe"] - common
        W = N_SINK + N_RECENT if case["window"] else 0
        share = (common + rest * (1.0 - (1.0 - left / max(rest, 1)) ** (T if case["lists"] == "own" else 1))) / case["B"]
        union, mine = (N - W) * share + W, (N - W) * case["nprobe"] / case["B"] + W
    small = 2 * S * Hkv * T * D * (4 if case["dtype"] == "f32" else 2)
    io = S * T * Hq * (D * (4 if case["dtype"] == "f32" else 2) + D * SIZE[case["out"]] + 4)
    return {"bytes": int(2 * D * e * S * Hkv * union) + small + io, "flops": int(4.0 * D * S * Hkv * R * mine)}
