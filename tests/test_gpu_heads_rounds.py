"""Bias, its gradient and dropout on value arrays of so many blocks that every wavefront takes several rounds of them."""
import numpy as np
import pytest

from gpu_util import to_dev_i32
from heads_ref import threefry
from test_gpu_heads import fs  # noqa: F401

pytestmark = pytest.mark.gpu


def many_blocks(rng, V):
    """CSR of a pattern whose value arrays take a wavefront of k_edges several rounds (2048 workgroups of four take 16 / V blocks each)."""
    M = K = 400000 if V == 4 else 300000
    deg = 8
    rows = np.repeat(np.arange(M, dtype=np.int64), deg)
    cols = rng.integers(0, K, rows.size)
    if V == 16:  # blocks of their own: 16 rows share few columns
        cols = (rows // 16 * 16 + rng.integers(0, 200, rows.size)) % K
    at = np.unique(rows * K + cols)
    return M, K, at // K, at % K


@pytest.mark.parametrize("V", [4, 8, 16])
def test_dropout_and_bias_over_many_rounds(fs, V):  # noqa: F811
    """Every wavefront takes several rounds: the kept entries are exactly those of the generator, biases exact, sums of whole numbers exact."""
    import torch
    p = 0.3
    rng = np.random.default_rng(V)
    M, K, rows, cols = many_blocks(rng, V)
    rp = to_dev_i32(np.concatenate([[0], np.cumsum(np.bincount(rows, minlength=M))]))
    fmt = fs.fs_convert(rp, to_dev_i32(cols), None, M, K, torch_dtype=torch.float16, V=V)
    assert fmt.n_blocks > 2048 * 4 * 16 // V, fmt.n_blocks
    state = torch.tensor([(3 << 33) + 5, 11], device="cuda")
    ones = torch.ones((2, fmt.V * fmt.nvec), dtype=torch.float16, device="cuda")
    got = fs.fs_edge_dropout(fmt, ones, fs.FsDropout(p, state))
    seed, step = state.tolist()
    key = threefry((seed & 0xFFFFFFFF, seed >> 32), step, 0, 20)
    factor = float(np.float16(np.float32(1 / (1 - p))))
    slot = fmt.csr_to_slot_t().long()
    outside = torch.ones(ones.shape[1], dtype=torch.bool, device="cuda")
    outside[slot] = False
    for h in range(2):
        word = threefry(threefry(key, h, 0, 20), rows, cols, 13)[0]
        want = np.where(word >= int(p * 2.0 ** 32), factor, 0.0)
        assert np.array_equal(fs.fs_blk_to_csr(fmt, got[h]).double().cpu().numpy(), want)
        assert not got[h][outside].any()
    n_buckets, reach = 24, 150
    lut = rng.integers(0, n_buckets, 2 * reach + 1).astype(np.uint8)
    table = rng.standard_normal((2, n_buckets)).astype(np.float16)
    bias = fs.FsBucketBias(torch.from_numpy(table).cuda(), torch.from_numpy(lut).cuda())
    bucket = lut[np.clip(cols - rows, -reach, reach) + reach]
    b = fs.fs_edge_bias(fmt, ones, bias, scale=0.0)
    for h in range(2):
        assert np.array_equal(fs.fs_blk_to_csr(fmt, b[h]).cpu().numpy(), table[h][bucket])
    g = rng.integers(-1, 2, (2, rows.size)).astype(np.float16)
    vals = torch.stack([fs.fs_csr_to_blk(fmt, torch.from_numpy(x).cuda()) for x in g])
    want = np.stack([np.bincount(bucket, weights=x.astype(np.float64), minlength=n_buckets) for x in g]).astype(np.float16)
    assert np.array_equal(fs.fs_edge_bias_backward(fmt, vals, bias).cpu().numpy(), want)
