"""tree_decode_attention's rows that attend values which are no numbers, or whose sums leave the range of fp32: they are computed
apart, and as exactly as all others.  Tolerances: test_gpu_tree.py."""
import math

import pytest
import torch

import paper_2502_08246_amd as saap
from test_gpu_tree import DEV, SCALE, Case
from test_gpu_tree_limits import _slot

pytestmark = pytest.mark.gpu
STEEP = torch.tensor([0.5, 0.25, 0.01, -0.03])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("T", [1, 3, 12])                # the shares added up by the last one; by a launch; rows of two waves
@pytest.mark.parametrize("lists", ["none", "shared", "own"])
def test_far_keys_and_steep_slopes_beside_a_value_that_is_no_number(dtype, T, lists):
    """One feature of a value that all rows attend; the other features, of scores of -10^5, keep what they have without it."""
    c = Case(dtype, 1, T, 4, 1, 500, 16, 16, lists, seed=5).cache()
    c.pos = c.pos + 200000
    c.compare(slopes=STEEP, drafts=False)
    bad = float("nan") if dtype == "fp8" else float("inf")
    c.Vd[0, 0, _slot(c, 0, 0, 497), 9] = 0x7f if dtype == "fp8" else bad
    c.V_held = c.V_held.clone()
    c.V_held[0, 0, 497, 9] = bad
    c.compare(slopes=STEEP, drafts=False)
    c.compare(torch.bfloat16, softcap=30.0, slopes=STEEP, drafts=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("lists,window", [("none", None), ("shared", None), ("shared", (1, 40))])
def test_lists_that_the_last_share_adds_up(dtype, lists, window):
    """Eight (sequence, head) pairs of eight rows: a list is taken as it is, and the share that ends last has the rows computed apart."""
    c = Case(dtype, 4, 2, 8, 2, 300, 16, 6, lists, window, seed=8, ragged=lists == "none").cache()
    c.n_keys = None
    c.seen = torch.ones_like(c.seen) if lists == "none" else c.seen
    c.pos = c.pos + 100000
    slopes = torch.tensor([0.5, 0.25, -0.125, 0.0, 0.5, 0.03, 0.25, 0.01])
    bad = float("nan") if dtype == "fp8" else float("inf")
    c.V_held = c.V_held.clone()
    for s, h in ((0, 0), (0, 1), (2, 1), (3, 0)):
        n = int(c.seen[s, h, 0].nonzero()[-1])           # the last key that is attended
        c.Vd[s, h, _slot(c, s, h, n), 77] = 0x7f if dtype == "fp8" else bad
        c.V_held[s, h, n, 77] = bad
    c.compare(slopes=slopes)
    c.compare(torch.bfloat16, slopes=slopes, drafts=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("T", [1, 3, 12])
@pytest.mark.parametrize("lists", ["none", "shared", "own"])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_values_at_the_end_of_the_range(dtype, T, lists, out):
    """Values of 2^125 to 2^127, all positive: their mean is such a number, their sum is none in fp32."""
    c = Case(dtype, 1, T, 4, 1, 500, 16, 16, lists, seed=6)
    c.q = c.q * 0.25                                     # many keys of about one weight
    c.V = ((c.V.float().abs() + 2.0).clamp(max=7.5) * 2.0 ** 124).to(c.V.dtype)
    c.vt = ((c.vt.float().abs() + 2.0).clamp(max=7.5) * 2.0 ** 124).to(c.vt.dtype)
    c.cache().compare(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
def test_a_value_in_one_tokens_own_bucket(dtype):
    """Token 0 alone lists bucket 0; a value there that is no number shows in its rows and in no other."""
    c = Case(dtype, 1, 5, 4, 1, 600, 16, 4, "own", seed=9)
    c.sel[0, :, 0] = torch.tensor([[0, 1, 2, 3], [1, 2, 3, 4], [5, 6, 7, 8], [1, 9, 10, 11], [12, 13, 14, 15]], dtype=torch.int32)
    member = torch.zeros(1, 5, 1, 16, dtype=torch.bool).scatter_(-1, c.sel.long(), True).transpose(1, 2)
    c.seen = member.gather(3, c.ids.long()[:, :, None].expand(-1, -1, 5, -1))
    c.cache()
    want, want_lse = c.run()
    c.compare()
    off, ln = int(c.off[0, 0, 0]), int(c.ln[0, 0, 0])
    assert ln > 1
    c.Vd[0, 0, off + 1, 3] = 0x7f if dtype == "fp8" else float("nan")
    got, lse = c.run()
    rest = [f for f in range(128) if f != 3]
    assert got[0, 0, :, 3].isnan().all() and torch.equal(got[0, 1:, :, 3], want[0, 1:, :, 3]) and torch.equal(lse, want_lse)
    assert torch.isfinite(got[..., rest]).all()
    c.V_held = c.V_held.clone()
    c.V_held[0, 0, int(c.idx[0, 0, off + 1]), 3] = float("nan")
    c.compare()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 12])
def test_scores_of_minus_infinity(dtype, T):
    """Such a key has no weight; a row with no other key is zero, its lse -inf.  One key of weight w: (w v) (1 / w) is three roundings of
    half a step 2^-24, and w v is the sum of the products of w's three parts in bf16, two more: 5 * 2^-24 of v."""
    c = Case(dtype, 1, T, 4, 1, 70, seed=7)
    c.q[..., 0] = -1.0
    c.K[0, 0, :-1, 0] = math.inf
    c.cache()
    call = lambda n: saap.dense_tree_decode_attention(c.q.to(DEV), c.Kd, c.Vd, SCALE, n_keys=torch.tensor([n], dtype=torch.int32, device=DEV))  # noqa: E731
    got, lse = call(70)
    v = c.Vd[0, 0, -1].double()
    assert ((got.double() - v).abs() <= 5 * 2.0 ** -24 * v.abs()).all() and torch.isfinite(lse).all()
    got, lse = call(69)
    assert (got == 0).all() and (lse == -math.inf).all()
