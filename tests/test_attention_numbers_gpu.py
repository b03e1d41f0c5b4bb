"""Attention over the paged cache at the edges of its numbers."""
import math

import numpy as np
import pytest
import torch

from oracle import verifier_oracle as VO
from test_verifier_gpu import _attend, _check, _np, _oracle, _setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Bn():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_03819_gb300 import binding
    binding.load_library()
    return binding


# new tokens per sequence: kernels for few rows and for many (groups of four rows per token)
FEW_AND_MANY = [1, 4, 17, 40]


@pytest.mark.parametrize("n", FEW_AND_MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_query_that_is_not_finite_gives_nan_in_its_row_alone(Bn, n, dtype, value):
    # its scores are infinities of both signs: cached keys have either, and the new tokens' keys are made to score -inf
    c = _setup(Bn, lens=[37, 300], n=n, heads=8, kv_heads=2, hd=64, page=16, dtype=dtype, seed=21, mask="causal")
    d = c["dims"]
    c["qkv"][:, :, d.heads, 5] = -1.0 if value == math.inf else 1.0
    want, want_lse, _ = _attend(Bn, c)
    assert want.isfinite().all()
    i = n - 1
    c["qkv"][:, i, 2, 5] = value                              # head 2 reads the keys' head 0
    out, lse, status = _attend(Bn, c)
    assert not status.any()
    assert out[:, i, 2].isnan().all() and lse[:, i, 2].isnan().all()
    rest = torch.ones_like(lse, dtype=torch.bool)
    rest[:, i, 2] = False
    assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], want_lse[rest])


@pytest.mark.parametrize("n", FEW_AND_MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lift", [-60, 0, 45, 100])
def test_pages_of_zeros_beside_values_of_any_scale(Bn, n, dtype, lift):
    # a page whose values are all zero has the scale that an append gives it, 2^-100; its tokens count in the sum as any others
    c = _setup(Bn, lens=[90, 160], n=n, heads=8, kv_heads=2, hd=64, page=16, dtype=dtype, seed=22, v_std=2.0 ** lift, nan_tail=False)
    c["vc"][::2], c["vs"][::2] = 0, 2.0 ** -100
    out, lse, status = _attend(Bn, c)
    assert not status.any()
    _check(c, out, lse)


@pytest.mark.parametrize("n", [1, 20])
def test_long_contexts_of_zeros(Bn, n):
    # keys and values of zeros, as a padded head has them: 32768 tokens of weight 1, and the new tokens, of whose keys the last row's
    # own alone meets its query, with a weight of 32768. Pieces of the work hold all of a sequence's cached tokens.
    b, hq, hkv, hd, page, length = 64, 8, 8, 64, 128, 32768
    pages = length // page
    d = Bn.CacheDims(batch=b, heads=hq, kv_heads=hkv, head_dim=hd, page=page, n_pages=b * pages, max_pages=pages)
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    kc, vc = z(b * pages, hkv, page, hd), z(b * pages, hkv, page, hd)
    ks = torch.full((b * pages, hkv), 2.0 ** -100, device="cuda")
    table = torch.arange(b * pages, dtype=torch.int32, device="cuda").view(b, pages)
    lens = torch.full((b,), length, dtype=torch.int32, device="cuda")
    q, k, v = (z(b, n, h, hd, dt=torch.bfloat16) for h in (hq, hkv, hkv))
    q[:, -1, :, 0], k[:, -1, :, 0] = 1.0, 1.0
    v[:, -1] = 3.0
    scale = math.log(length)                                  # a score of log 32768
    out, lse, status = z(b, n, hq, hd, dt=torch.bfloat16), z(b, n, hq, dt=torch.float32), z(b, dt=torch.int32)
    Bn.tf_tree_attention(d, q, k, v, kc, vc, ks, ks.clone(), table, lens, None, scale, out, lse, status, Bn.alloc_attention_workspace(d, n))
    torch.cuda.synchronize()
    assert not status.any()
    seen = length + torch.arange(1, n + 1, dtype=torch.float64)   # tokens of weight 1
    seen[-1] += length - 1
    # sums of 32768 terms in fp32, and one weight of a score of 10
    assert (lse.cpu().double() - seen.log()[None, :, None]).abs().max() <= (length + 16) * 2.0 ** -24
    want = torch.zeros(n, dtype=torch.float64)
    want[-1] = 3.0 * length / seen[-1]
    assert (out.cpu().double() - want[None, :, None, None]).abs().max() <= 3.0 * 2.0 ** -8


def _equal_scores(Bn, n, dtype, length, power):
    """Every key is the same, so that every score is -2^power times the row's own factor and every weight 1: the output is the mean of
    the values and lse the score, whatever page and scale a token lies in."""
    c = _setup(Bn, lens=[length, max(length - 7, 0)], n=n, heads=8, kv_heads=2, hd=64, page=16, dtype=dtype, seed=23, mask="causal", nan_tail=False)
    d = c["dims"]
    c["kc"][:], c["ks"][:] = VO.to_e4m3(np.float64(1.0)), 2.0 ** -3
    c["qkv"][:, :, :d.heads] = -1.0 - 0.25 * torch.arange(d.heads)[:, None] / d.heads
    c["qkv"][:, :, d.heads:d.heads + d.kv_heads] = 2.0 ** -3
    c["scale"] = 2.0 ** (power - 3)                           # 64 products of 2^-3 each
    out, lse, status = _attend(Bn, c)
    assert not status.any()
    o, l, mag, _ = _oracle(c)
    terms = length + n
    # equal scores have equal weights in any arithmetic that rounds them alike; the rest are the sums, a weight's rounding and the output's.
    # A score is a sum of head_dim products in fp32.
    r = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    tol = mag * (r + (2 * terms + 16) * 2.0 ** -24) + r * np.abs(o)
    assert (np.abs(_np(out) - o) <= tol).all(), float((np.abs(_np(out) - o) / tol).max())
    assert (np.abs(_np(lse) - l) <= (d.head_dim + 16) * 2.0 ** -24 * np.abs(l) + (terms + 16) * 2.0 ** -24).all()


@pytest.mark.parametrize("n", FEW_AND_MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [0, 40, 300])
@pytest.mark.parametrize("power", [7, 10])
def test_rows_whose_scores_are_all_far_below_zero(Bn, n, dtype, length, power):
    _equal_scores(Bn, n, dtype, length, power)


@pytest.mark.parametrize("n", FEW_AND_MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [0, 40, 300])
@pytest.mark.parametrize("power", [20, 25])
def test_equal_scores_where_fp32_is_coarse(Bn, n, dtype, length, power):
    _equal_scores(Bn, n, dtype, length, power)


@pytest.mark.parametrize("n", FEW_AND_MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [0, 40, 300])
@pytest.mark.parametrize("power", [99, 101, 124])
def test_rows_whose_scores_lie_around_and_below_minus_1e30(Bn, n, dtype, length, power):
    _equal_scores(Bn, n, dtype, length, power)


# contexts with new tokens alone, with few rows and with many
SHAPES = [([0, 0], 64, 128), ([0], 130, 64), ([0, 0, 0], 3, 64), ([700, 130], 1, 128), ([300, 5], 4, 64), ([700, 64, 1], 33, 128), ([900], 20, 64)]


@pytest.mark.parametrize("lens,n,hd", SHAPES)
@pytest.mark.parametrize("mask", ["causal", "tree"])
@pytest.mark.parametrize("q_std", [0.5, 3.0])
def test_bf16_outputs_to_what_their_arithmetic_leaves(Bn, lens, n, hd, mask, q_std):
    """A score is an fp32 sum of head_dim exact products, each sum cut to fp32: (hd + 16) 2^-23 of the largest sum of |q_d k_td|, with 16 for the
    scalings, the exponential and its argument. Many rows hold their queries in two e4m3 parts over cached keys: 2^-17 of the row's
    largest element for each element. A weight is then off by twice that, and by its rounding: f16 over cached tokens (2^-11, and
    2^-25 absolute where the largest is 2^7 at least, times 448 scales), two bf16 parts or fp32 over new ones (2^-16). Sums of t terms
    in fp32 lose t 2^-24 each; the output is rounded to bf16 once, 2^-8."""
    c = _setup(Bn, lens=lens, n=n, heads=8, kv_heads=2, hd=hd, page=32, mask=mask, seed=31, q_std=q_std)
    d = c["dims"]
    out, lse, status = _attend(Bn, c)
    assert not status.any()
    o, l, mag, top = _oracle(c)
    x = _np(c["qkv"])
    q_top = np.abs(x[:, :, :8]).max(-1)
    keys = np.abs(VO.from_e4m3(c["kc"]) * c["ks"][:, :, None, None]).sum(-1)
    split = q_top * np.nanmax(keys, initial=0.0) * c["scale"] * 2.0 ** -17 if max(lens) else 0.0
    z = (hd + 16) * 2.0 ** -23 * top + split
    terms = max(lens) + n
    r = (2.0 ** -11 if max(lens) else 0.0) + 2.0 ** -16
    small = terms * 2.0 ** -32 * 448 * float(c["vs"].max()) if max(lens) else 0.0
    tol = mag * (2 * z[..., None] + r + (2 * terms + 16) * 2.0 ** -24) + small + 2.0 ** -8 * (1 + 2.0 ** -7) * np.abs(o) + 1e-30
    assert (np.abs(_np(out) - o) <= tol).all(), float((np.abs(_np(out) - o) / tol).max())
    fin = np.isfinite(l)
    assert (np.abs(_np(lse) - l)[fin] <= (2 * z + (terms + 16) * 2.0 ** -24)[fin] + 2.0 ** -22 * (1 + np.abs(l[fin]))).all()
