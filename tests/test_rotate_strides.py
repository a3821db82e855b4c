"""Strides between tokens that norm_rotate takes and refuses: a multiple of 16 bytes, whatever the type."""
import ctypes

import pytest
import torch

import paper_2502_08246_amd as saap
from test_drafted_host import A, BIG, _rotation

DEV = "cuda:0"


@pytest.mark.parametrize("stride,dtype,taken", [(1028, 0, True), (1024, 0, True), (1026, 0, False), (1025, 0, False), (1032, 1, True), (1028, 1, False)])
def test_which_strides_are_taken(stride, dtype, taken):
    """A head size that is refused later than strides are says that this stride was none of the reasons."""
    lib = saap.load_library()
    r = _rotation(Hq=8, q_stride=1024, k_stride=stride, dtype=dtype)
    small = _rotation(Hq=8, q_stride=1024, k_stride=stride, dtype=dtype, d=64)
    if not taken:
        assert lib.saap_norm_rotate(ctypes.byref(r), *A[4:10], None) == -1
        assert lib.saap_norm_rotate_grads(ctypes.byref(r), *A[4:14], A[14], BIG, None) == -1
    want = -2 if taken else -1
    assert lib.saap_norm_rotate(ctypes.byref(small), *A[4:10], None) == want
    assert lib.saap_norm_rotate_grads(ctypes.byref(small), *A[4:14], A[14], BIG, None) == want


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gap", [(torch.float32, 4), (torch.float32, 20), (torch.bfloat16, 8), (torch.bfloat16, 24)])
def test_rows_a_few_elements_apart(dtype, gap):
    """Tokens 16 bytes and more behind the end of the one before: the bits that the same rows have side by side."""
    g = torch.Generator().manual_seed(gap)
    S, T, Hq, Hkv = 2, 37, 6, 2
    def apart(H):
        rows = torch.full((S, T, H * 128 + gap), float("nan"), dtype=dtype)
        rows[..., :H * 128] = torch.randn(S, T, H * 128, generator=g).to(dtype)
        return rows.to(DEV)[..., :H * 128].unflatten(2, (H, 128))
    q, k = apart(Hq), apart(Hkv)
    assert q.stride(1) == Hq * 128 + gap and k.stride(1) == Hkv * 128 + gap
    pos = torch.randint(0, 9999, (S, T), generator=g).to(torch.int32).to(DEV)
    freqs, w = saap.rotary_frequencies(128, device=DEV), (1 + 0.1 * torch.randn(128, generator=g)).to(DEV)
    far, near = saap.norm_rotate(q, k, pos, freqs, w, w), saap.norm_rotate(q.contiguous(), k.contiguous(), pos, freqs, w, w)
    assert all(torch.equal(a, b) for a, b in zip(far, near)) and torch.isfinite(far[0]).all()
    grads = [torch.randn(t.shape, generator=g).to(dtype).to(DEV) for t in near]
    far, near = (saap.norm_rotate_grads(a, b, pos, freqs, *grads, w, w) for a, b in ((q, k), (q.contiguous(), k.contiguous())))
    assert all(torch.equal(a, b) for a, b in zip(far, near)) and all(torch.isfinite(t).all() for t in far)
