"""What the calls for drafted tokens refuse before they touch a device, and their host-side helpers."""
import ctypes
import math

import pytest
import torch

import paper_2502_08246_amd as saap
from paper_2502_08246_amd import binding

I, P, F = ctypes.c_int32, ctypes.c_void_p, ctypes.c_float
BIG = ctypes.c_size_t(1 << 34)
A = [P(4096 * (i + 1)) for i in range(16)]      # aligned addresses that nothing may use
ODD = P(4100)


class Rotation(ctypes.Structure):
    _fields_ = [("positions", P), ("freqs", P), ("q_weight", P), ("k_weight", P), ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64)] + \
        [(n, I) for n in ("S", "T", "Hq", "Hkv", "d", "rot", "pairs", "norm", "weight_per_head", "dtype")] + [("eps", F), ("magnitude", F)]


class Tree(ctypes.Structure):
    _fields_ = [(n, P) for n in ("tree", "k_tree", "v_tree", "idx", "slopes", "pos", "starts")] + \
        [(n, I) for n in ("S", "T", "Hq", "Hkv", "d")] + [("scale", F), ("softcap", F)]


@pytest.fixture(scope="module")
def lib():
    return saap.load_library()


def _rotation(**kw):
    a = dict(positions=A[0], freqs=A[1], q_weight=A[2], k_weight=A[3], q_stride=6144, k_stride=6144, S=2, T=3, Hq=32, Hkv=8, d=128, rot=128,
             pairs=0, norm=1, weight_per_head=0, dtype=1, eps=1e-6, magnitude=1.0)
    a.update(kw)
    return Rotation(**a)


@pytest.mark.parametrize("kw,status", [
    (dict(positions=None), -1), (dict(freqs=None), -1), (dict(S=0), -1), (dict(T=0), -1), (dict(Hq=0), -1), (dict(Hkv=-1), -1), (dict(dtype=2), -1),
    (dict(rot=0), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(norm=0), -1), (dict(q_stride=4095), -1), (dict(q_stride=4096 + 4), -1),
    (dict(k_stride=1016), -1), (dict(k_stride=1028, dtype=0), None), (dict(k_stride=1026, dtype=0), -1), (dict(q_weight=ODD), -1),
    (dict(d=64), -2), (dict(rot=130), -2), (dict(rot=24), -2), (dict(rot=144), -2), (dict(S=1 << 20, T=1 << 12), -2), (dict(S=1, T=(1 << 25) + 1), -2), (dict(Hq=5000, q_stride=640000), -2),
])
def test_norm_rotate_refuses(lib, kw, status):
    if status is None:
        return                                  # a stride that fp32 allows: nothing to refuse, and no device to run on
    r = _rotation(**kw)
    assert lib.saap_norm_rotate(ctypes.byref(r), *A[4:10], None) == status
    assert lib.saap_norm_rotate_grads(ctypes.byref(r), *A[4:14], A[14], BIG, None) == status


def test_norm_rotate_refuses_what_does_not_go_together(lib):
    r = ctypes.byref(_rotation())
    assert lib.saap_norm_rotate(None, *A[4:10], None) == -1
    assert lib.saap_norm_rotate(r, None, None, *A[6:10], None) == -1
    assert lib.saap_norm_rotate(r, None, A[5], A[6], None, A[8], None, None) == -1         # an output without its tensor
    assert lib.saap_norm_rotate(r, A[4], A[5], None, None, A[8], A[9], None) == -1         # a tensor without outputs
    assert lib.saap_norm_rotate(r, ODD, *A[5:10], None) == -1
    assert lib.saap_norm_rotate(r, A[4], A[5], A[6], ODD, A[8], A[9], None) == -1
    def grads(**kw):
        a = dict(q=A[4], k=A[5], gqf=A[6], gqr=A[7], gkf=A[8], gkr=A[9], dq=A[10], dk=A[11], dqw=A[12], dkw=A[13], ws=A[14], n=BIG)
        a.update(kw)
        return lib.saap_norm_rotate_grads(r, a["q"], a["k"], a["gqf"], a["gqr"], a["gkf"], a["gkr"], a["dq"], a["dk"], a["dqw"], a["dkw"],
                                          a["ws"], a["n"], None)
    assert grads(dq=None) == -1 and grads(q=None) == -1 and grads(gqf=None, gqr=None) == -1 and grads(dqw=None) == -1
    assert grads(ws=None) == -1 and grads(gkr=ODD) == -1 and grads(n=ctypes.c_size_t(65536)) == -3


def _attend(lib, which="lists", tree=None, **kw):
    t = dict(tree=A[0], k_tree=A[1], v_tree=A[2], idx=A[3], slopes=None, pos=None, starts=None, S=2, T=5, Hq=8, Hkv=2, d=128, scale=0.1, softcap=0.0)
    t.update(tree or {})
    a = dict(q=A[4], K=A[5], V=A[6], ks=A[7], vs=A[8], off=A[9], ln=A[10], sel=A[11], nprobe=3, per=1, res=-1, out=A[12], odt=0, lse=A[13], rows=100,
             runs=16, dt=1, ws=A[14], n=BIG, n_keys=None)
    a.update(kw)
    r = ctypes.byref(Tree(**t))
    tail = (a["ws"], a["n"], None)
    lists = (a["off"], a["ln"], a["sel"], I(a["nprobe"]), I(a["per"]), I(a["res"]), a["out"], I(a["odt"]), a["lse"], I(a["rows"]), I(a["runs"]))
    dense = (a["n_keys"], a["out"], I(a["odt"]), a["lse"], I(a["rows"]))
    if which == "lists":
        return lib.saap_tree_decode_attention(r, a["q"], a["K"], a["V"], *lists, I(a["dt"]), *tail)
    if which == "lists8":
        return lib.saap_tree_decode_attention_fp8(r, a["q"], a["K"], a["V"], a["ks"], a["vs"], *lists, *tail)
    if which == "dense":
        return lib.saap_dense_tree_decode_attention(r, a["q"], a["K"], a["V"], *dense, I(a["dt"]), *tail)
    return lib.saap_dense_tree_decode_attention_fp8(r, a["q"], a["K"], a["V"], a["ks"], a["vs"], *dense, *tail)


EVERY = [(dict(q=None), -1), (dict(K=None), -1), (dict(V=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(q=ODD), -1), (dict(out=ODD), -1),
         (dict(odt=2), -1), (dict(rows=0), -1), (dict(rows=1 << 23), -2), (dict(n=ctypes.c_size_t(1 << 16)), -3),
         (dict(tree=dict(S=0)), -1), (dict(tree=dict(T=0)), -1), (dict(tree=dict(Hq=7)), -1), (dict(tree=dict(d=64)), -2), (dict(tree=dict(T=65)), -2),
         (dict(tree=dict(Hq=6)), -2), (dict(tree=dict(Hq=32)), -2), (dict(tree=dict(S=2049)), -2), (dict(tree=dict(k_tree=None)), -1),
         (dict(tree=dict(tree=None)), -1), (dict(tree=dict(v_tree=None)), -1), (dict(tree=dict(k_tree=ODD)), -1), (dict(tree=dict(slopes=A[15])), -1),
         (dict(tree=dict(softcap=-1.0)), -1), (dict(tree=dict(softcap=math.inf)), -1), (dict(tree=dict(softcap=math.nan)), -1)]
LISTS = [(dict(off=None), -1), (dict(ln=None), -1), (dict(sel=None), -1), (dict(nprobe=-1), -1), (dict(nprobe=17), -1), (dict(runs=0), -1),
         (dict(res=16), -1), (dict(res=-2), -1), (dict(runs=8194), -2), (dict(tree=dict(starts=A[15], idx=None)), -1),
         (dict(tree=dict(slopes=A[15], pos=A[15], idx=None)), -1)]


@pytest.mark.parametrize("which", ["lists", "lists8", "dense", "dense8"])
def test_tree_attention_refuses(lib, which):
    for kw, status in EVERY + (LISTS if which.startswith("lists") else []):
        assert _attend(lib, which, **kw) == status, kw
    if which.endswith("8"):
        assert _attend(lib, which, ks=None) == -1 and _attend(lib, which, vs=None) == -1
    else:
        assert _attend(lib, which, dt=2) == -1


def _accept(lib, fp8=False, **kw):
    a = dict(ids=A[0], k=A[1], v=A[2], path=A[3], pos=A[4], off=A[5], ln=A[6], idx=A[7], K=A[8], V=A[9], ks=A[10], vs=A[11], res=A[12], flag=A[13], S=2,
             Hkv=2, T=9, P=4, Ncap=200, B=16, d=128, dt=1, sink=1, recent=31)
    a.update(kw)
    head = [a[n] for n in ("ids", "k", "v", "path", "pos", "off", "ln", "idx", "K", "V")]
    sizes = [I(a[n]) for n in ("S", "Hkv", "T", "P", "Ncap", "B", "d")]
    tail = [I(a["sink"]), I(a["recent"]), None]
    if fp8:
        return lib.saap_append_accepted_fp8(*head, a["ks"], a["vs"], a["res"], a["flag"], *sizes, *tail)
    return lib.saap_append_accepted(*head, a["res"], a["flag"], *sizes, I(a["dt"]), *tail)


@pytest.mark.parametrize("fp8", [False, True])
def test_append_accepted_refuses(lib, fp8):
    for n in ("ids", "k", "v", "path", "off", "ln", "idx", "K", "V", "flag") + (("ks", "vs") if fp8 else ()):
        assert _accept(lib, fp8, **{n: None}) == -1, n
    for n in ("k", "v", "K", "V"):
        assert _accept(lib, fp8, **{n: ODD}) == -1, n
    for n in ("S", "Hkv", "T", "P", "Ncap", "B"):
        assert _accept(lib, fp8, **{n: 0}) == -1, n
    assert _accept(lib, fp8, pos=None) == -1                     # a window needs positions
    assert _accept(lib, fp8, sink=-1) == -1 and _accept(lib, fp8, recent=200) == -1
    assert _accept(lib, fp8, res=None) == -1                     # a window without its ids
    assert _accept(lib, fp8, d=64) == -2 and _accept(lib, fp8, B=8193) == -2 and _accept(lib, fp8, P=65, recent=100) == -2
    assert _accept(lib, fp8, P=32) == -2                         # more than the ring
    if not fp8:
        assert _accept(lib, dt=2) == -1


def test_python_calls_look_at_what_they_read():
    x = torch.zeros(1, 2, 4, 128)
    pos, f = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(64, dtype=torch.float64)
    with pytest.raises(ValueError):
        saap.norm_rotate(None, None, pos, f)
    with pytest.raises(ValueError):
        saap.norm_rotate(x, x, pos, f)                           # host memory
    with pytest.raises(ValueError):
        saap.tree_decode_attention(x[0], x, x, pos, pos, pos, 1.0)
    with pytest.raises(ValueError):
        saap.append_accepted(pos, x, x, pos, None, pos, pos, pos, x, x)
    with pytest.raises(TypeError):
        saap.dense_tree_decode_attention_fp8(x, x, x, f, f, 1.0)  # not an 8-bit cache


def test_workspace_sizes():
    sized = lambda **kw: saap.workspace_bytes(binding.OP_TREE_DECODE_ATTENTION, **kw)  # noqa: E731
    base = dict(S=1, Hq=32, Hkv=8, N=4, dtype=1)
    assert sized(**base) > 0
    assert sized(**base, B=1024, nprobe=51, mode=1) > sized(**base, B=1024, nprobe=51) > sized(**base)
    assert sized(**{**base, "Hq": 30}) == 0 and sized(**{**base, "N": 65}) == 0 and sized(**{**base, "S": 0}) == 0
    assert saap.workspace_bytes(binding.OP_NORM_ROTATE_GRADS, S=1, Hq=8, Hkv=0, N=100) > 0
    assert saap.workspace_bytes(binding.OP_NORM_ROTATE_GRADS, S=1, Hq=0, Hkv=0, N=100) == 0


def test_frequencies():
    want = torch.tensor([500000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    plain = saap.rotary_frequencies(64, device="cpu")
    assert plain.dtype == torch.float64 and torch.allclose(plain, want, rtol=1e-14)
    assert torch.equal(saap.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu"), plain / 4)
    base = saap.rotary_frequencies(64, scaling="base", factor=4.0, device="cpu")
    assert base[0] == 1.0 and math.isclose(float(base[-1]), float(plain[-1]) / 4, rel_tol=1e-12)
    bands = saap.rotary_frequencies(64, scaling="bands", factor=8.0, context=8192, device="cpu")
    turns = 8192 * plain / (2 * math.pi)
    assert torch.equal(bands[turns > 4], plain[turns > 4]) and torch.allclose(bands[turns < 1], plain[turns < 1] / 8, rtol=1e-14)
    between = (turns > 1) & (turns < 4)
    assert between.any() and ((bands < plain) & (bands > plain / 8))[between].all()
    for bad in (dict(rot=7), dict(rot=0), dict(rot=64, factor=0.0), dict(rot=64, scaling="other"), dict(rot=64, scaling="bands", low=4.0)):
        with pytest.raises(ValueError):
            saap.rotary_frequencies(**bad, device="cpu")


def test_masks_of_trees():
    parents = torch.tensor([[-1, 0, 0, 2, 1], [-1, -1, 1, 5, 5]])
    assert saap.tree_masks(parents).tolist() == [[1, 3, 5, 13, 19], [1, 2, 6, 0, 0]]
    chain = saap.tree_masks(torch.arange(-1, 63)[None])
    assert chain[0, 62] == 2 ** 63 - 1 and chain[0, 63] == -1
    for bad in (torch.tensor([[0]]), torch.tensor([[-1, 1]]), torch.zeros(1, 65, dtype=torch.int64), torch.zeros(3)):
        with pytest.raises(ValueError):
            saap.tree_masks(bad)
