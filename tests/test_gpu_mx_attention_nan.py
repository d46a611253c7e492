"""NaNs on either side of the joined attention: a NaN log sum, a NaN key or
value, and a NaN in the earlier result are never taken for a query without
keys, over every kernel (few rows, four and eight waves, a block an item and
shared items with their joining launch)."""

import numpy as np
import pytest
import torch

from paper_2607_20940_amd import mssa

from lowbit_common import cuda, f64
from test_gpu_mx_attention import _cache

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
# tokens of a cache that one block reads whole, and of one that several share
TOKENS = [100, 3000]
ROWS = [1, 20, 300, 2100]


def _attend(q, k, v, lens, prior=None):
    B, n, H, D = q.shape
    T, KH = k[0].shape[1:3]
    d = mssa.mx_attention_desc(B, n, H, KH, D, T)
    ws = torch.empty(max(16, mssa.mssa_mx_attention_workspace_size(d)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    lse = torch.empty(B, H, n, device="cuda")
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    mssa.mssa_mx_attention(d, q, k[0], k[1], v[0], v[1], kv_len, *(prior or (None, None)), ws, out, lse)
    torch.cuda.synchronize()
    return out, lse


def _inputs(n, T, B=3, H=2, D=64):
    rng = np.random.default_rng(n + T)
    q, po = (cuda(rng.normal(size=(B, n, H, D)), "bf16") for _ in range(2))
    k, v = (list(_cache(rng, B, T, H, D)[:2]) for _ in range(2))
    pl = cuda(rng.normal(size=(B, H, n)), "f32")
    return q, k, v, po, pl


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("T", TOKENS)
def test_nan_prior_log_sum(n, T):
    """An earlier log sum of NaN makes its query's output and log sum NaN, over an empty cache and a full one."""
    q, k, v, po, pl = _inputs(n, T)
    pl[:, 1, n - 1] = NAN
    out, lse = _attend(q, k, v, [0, T, 65], (po, pl))
    want = np.zeros((3, 2, n), bool)
    want[:, 1, n - 1] = True
    assert np.array_equal(np.isnan(f64(lse)), want)
    assert np.array_equal(np.isnan(f64(out)), np.broadcast_to(want.transpose(0, 2, 1)[..., None], out.shape))


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("T", TOKENS)
def test_nan_key_with_a_prior_without_keys(n, T):
    """A NaN key next to a prior without keys: NaN output and log sum, and a further join keeps them."""
    q, k, v, po, pl = _inputs(n, T)
    k[1][1, T // 2, 0, 1] = 255
    pl[:] = -INF
    out, lse = _attend(q, k, v, [T, T, 0], (po, pl))
    want = np.zeros((3, 2, n), bool)
    want[1, 0] = True
    assert np.array_equal(np.isnan(f64(lse)), want)
    wide = np.broadcast_to(want.transpose(0, 2, 1)[..., None], out.shape)
    assert np.array_equal(np.isnan(f64(out)), wide)
    assert np.isneginf(f64(lse)[2]).all() and (f64(out)[2] == 0).all()
    clean = _inputs(n, T)
    again, lse2 = _attend(q, clean[1], clean[2], [T, T, T], (out, lse))
    assert np.array_equal(np.isnan(f64(lse2)), want)
    assert np.array_equal(np.isnan(f64(again)), wide)


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("T", TOKENS)
def test_nan_prior_output(n, T):
    """A NaN in an earlier output stays, also where its share of the joint softmax is below fp32's smallest number;
    what an earlier result without keys holds is not used."""
    q, k, v, po, pl = _inputs(n, T)
    po[0, 0, 1, 3] = NAN
    po[1, n - 1, 0, 63] = NAN
    pl[1] = -500.0
    po[2, 0, 0] = NAN
    pl[2] = -INF
    out, lse = _attend(q, k, v, [T, T, T], (po, pl))
    want = np.zeros(out.shape, bool)
    want[0, 0, 1, 3] = want[1, n - 1, 0, 63] = True
    assert np.array_equal(np.isnan(f64(out)), want)
    assert np.isfinite(f64(lse)).all()
