"""append_accepted where some of the accepted tokens are refused: a window that is still filling keeps its keys together, and positions
below zero are refused as the calls for single tokens refuse them.  Bit by bit against those calls."""
import pytest
import torch

import paper_2502_08246_amd as saap
from test_gpu_accept import DEV, _index, _one_by_one

pytestmark = pytest.mark.gpu
NAMES = ("off", "len", "idx", "Ks", "Vs", "resident_ids")


def _start(kind, S, Hkv, N, B, window, T, seed):
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    g, rand, cent, index = _index(S, Hkv, N, B, 20, dtype, window, seed)
    x, k, v = rand(S, Hkv, T, 128), rand(S, Hkv, T, 128), rand(S, Hkv, T, 128)
    scales = ()
    if kind == "fp8":
        index[3], index[4], *scales = saap.quantize_kv(index[3], index[4])
    return cent, index, x, k, v, tuple(scales)


def _accept(ids, k, v, path, pos, index, scales, window, flag=None):
    call = saap.append_accepted_fp8 if scales else saap.append_accepted
    more = {} if window is None else dict(resident_ids=index[5], n_sink=window[0], n_recent=window[1])
    return call(ids, k, v, path, pos, *index[:5], *scales, overflow_flag=flag, **more)


def _push(cent, index, x, k, v, s, h, token, position, window, scales):
    """window_push of one token of one head."""
    at = lambda t: t[s:s + 1, h:h + 1].contiguous()  # noqa: E731
    row = lambda t: t[s:s + 1, h:h + 1, token].contiguous()  # noqa: E731
    own = [at(t) for t in index]
    call = saap.window_push_fp8 if scales else saap.window_push
    call(row(x), row(k), row(v), torch.tensor([position], dtype=torch.int32, device=DEV), cent[h:h + 1].contiguous(), None, *own[:5],
         *(at(t) for t in scales), own[5], *window)
    for t, one in zip(index, own):
        t[s:s + 1, h:h + 1] = one


# N keys held, sink + recent slots, tokens of a path, where a bucket id is none
FILLING = [(10, (4, 16), 6, [2]), (10, (4, 16), 6, [0]), (10, (4, 16), 6, [5]), (17, (4, 16), 6, [1]), (17, (4, 16), 9, [2, 4]),
           (19, (4, 16), 5, [0]), (18, (4, 16), 6, [3]), (3, (6, 0), 5, [1]), (4, (0, 30), 30, [7, 20])]


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("N,window,P,bad", FILLING)
def test_a_filling_window_has_no_holes(N, window, P, bad, kind):
    """Head 1 of sequence 0 has ids that are none: of the keys that fill its window those before the first such key are stored, of the
    others (whose slots are the ring's) all with an id; the other heads store every key."""
    S, Hkv, B, W = 2, 2, 16, window[0] + window[1]
    cent, index, x, k, v, scales = _start(kind, S, Hkv, N, B, window, P, seed=N + P)
    ids = saap.assign_keys(x, cent)
    for i, t in enumerate(bad):
        ids[0, 1, t] = (-1, B)[i % 2]
    path = torch.arange(P, dtype=torch.int32, device=DEV).expand(S, P).contiguous()
    theirs = [t.clone() for t in index]
    stored = {}
    for s in range(S):
        for h in range(Hkv):
            holes = bad if (s, h) == (0, 1) else []
            stored[s, h] = [t for t in range(P) if t not in holes and (N + t >= W or not any(b < t for b in holes))]
            for t in stored[s, h]:
                _push(cent, theirs, x, k, v, s, h, t, N + t, window, scales)
    flag = _accept(ids, k, v, path, torch.full((S,), N, dtype=torch.int32, device=DEV), index, scales, window)
    assert int(flag[0]) == 1
    for name, a, b in zip(NAMES, index, theirs):
        assert torch.equal(a, b), name
    held = index[1][0, 1, B]
    assert int(held) == N + sum(N + t < W for t in stored[0, 1])
    base = int(index[0][0, 1, B])
    assert (index[2][0, 1, base:base + int(held)] >= 0).all()


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_a_filling_window_takes_the_next_position_only(kind):
    """After a refused key the caller's positions run ahead of the window: such keys are refused, and taken when they are the next."""
    N, window, T = 10, (4, 16), 4
    cent, index, x, k, v, scales = _start(kind, 1, 2, N, 16, window, T, seed=9)
    ids = saap.assign_keys(x, cent)
    path = torch.arange(T, dtype=torch.int32, device=DEV)[None]
    before = [t.clone() for t in index]
    for first in (N + 1, N - 1, 0, N + 5):
        flag = _accept(ids, k, v, path, torch.tensor([first], dtype=torch.int32, device=DEV), index, scales, window)
        assert int(flag[0]) == 1, first
        for name, a, b in zip(NAMES, index, before):
            assert torch.equal(a, b), (first, name)
    flag = _accept(ids, k, v, path, torch.tensor([N], dtype=torch.int32, device=DEV), index, scales, window)
    assert int(flag[0]) == 0 and index[1][0, :, 16].tolist() == [N + T] * 2


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("window", [None, (0, 0)])
@pytest.mark.parametrize("first", [-1, -3, -100, 2 ** 31 - 3])
def test_positions_below_zero_are_refused(first, window, kind):
    N, T, P = 200, 9, 6
    cent, index, x, k, v, scales = _start(kind, 2, 2, N, 16, window, T, seed=11)
    path = torch.tensor([[0, 3, 5, 8, 1, 2], [4, 4, 6, -1, 0, 0]], dtype=torch.int32, device=DEV)
    pos = torch.tensor([first, N], dtype=torch.int32, device=DEV)
    theirs = [None if t is None else t.clone() for t in index]
    want = _one_by_one(theirs, cent, x, k, v, path, pos, window, scales)
    flag = _accept(saap.assign_keys(x, cent), k, v, path, pos, index, scales, window)
    assert int(flag[0]) == int(want[0]) == 1
    for name, a, b in zip(NAMES, index, theirs):
        assert a is None or torch.equal(a, b), name
