"""Attention with heads, a bucket bias and dropout on the GPU, forward and backward, against the 64-bit reference; and the same
steps on value arrays.  The bounds come from the reference (half steps of the element type, fp32 sums)."""
import ctypes

import numpy as np
import pytest

from gpu_util import to_dev_i32, torch_dtype
from heads_ref import FLOOR, HALF_STEP, Attention, bucket_of, keep_factors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fs():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2412_11007_amd as fs
    fs.load_library()
    return fs


def stored_of(rng, M, K, kind):
    if kind == "band":  # a sequence: the last 40 columns and the first two
        i, j = np.arange(M)[:, None], np.arange(K)[None]
        return (j <= i) & ((i - j < 40) | (j < 2))
    if kind == "dense":
        return np.ones((M, K), dtype=bool)
    if kind == "empty":
        return np.zeros((M, K), dtype=bool)
    s = rng.random((M, K)) < 0.12
    s[rng.random(M) < 0.2] = False
    s[:, rng.random(K) < 0.2] = False
    if kind == "hub":  # rows and columns that are cut into parts
        s[M // 3] = True
        s[:, K // 2] = True
    return s


def csr_of(stored):
    rows, cols = np.nonzero(stored)
    rp = np.concatenate([[0], np.cumsum(np.bincount(rows, minlength=stored.shape[0]))])
    return to_dev_i32(rp), to_dev_i32(cols)


class Problem:
    def __init__(self, fs, seed, M, K, heads, kv, d, N, dtype, kind="random", p=0.0, bias=None, shift=0, V=0, V_t=0, chunk=0, layout="rows"):
        import torch
        rng = np.random.default_rng(seed)
        self.fs, self.dt, self.dtype = fs, torch_dtype(dtype), dtype
        self.stored = stored_of(rng, M, K, kind)
        rp, ci = csr_of(self.stored)
        self.fmt = fs.fs_convert(rp, ci, None, M, K, torch_dtype=self.dt, V=V, chunk=chunk)
        rpt, cit, _ = fs.fs_csr_transpose(rp, ci, M, K)
        self.fmt_t = fs.fs_convert(rpt, cit, None, K, M, torch_dtype=self.dt, V=V_t, chunk=chunk)

        def operand(rows, h, width):
            t = torch.from_numpy(rng.standard_normal((rows, h, width))).to(self.dt).cuda()
            if layout == "rows":
                return t
            if layout == "heads":  # (heads, rows, width) in memory
                return t.transpose(0, 1).contiguous().transpose(0, 1)
            wide = torch.full((rows, h, width + 24), 9.0, dtype=self.dt, device="cuda")  # a column range of something wider
            wide[:, :, 8:8 + width] = t
            return wide[:, :, 8:8 + width]

        self.X, self.Y, self.H, self.G = operand(M, heads, d), operand(K, kv, d), operand(K, kv, N), operand(M, heads, N)
        self.scale = d ** -0.5
        self.state = torch.tensor([seed * 0x123456789 + 1, 3], device="cuda")
        self.drop = fs.FsDropout(p, self.state) if p else None
        self.bias = None
        extra = {}
        if bias:
            n, reach = bias
            buckets = torch.from_numpy(rng.integers(0, n, 2 * reach + 1).astype(np.uint8)).cuda()
            self.bias = fs.FsBucketBias(torch.from_numpy(rng.standard_normal((heads, n))).to(self.dt).cuda(), buckets, shift=shift)
            extra = dict(table=self.f64(self.bias.table), buckets=buckets.cpu().numpy(), shift=shift)
        self.ref = Attention(self.stored, self.f64(self.X), self.f64(self.Y), self.f64(self.H), self.scale, p=p, state=self.state.tolist(), dtype=dtype, **extra)

    @staticmethod
    def f64(t):
        return t.double().cpu().numpy()

    def forward(self, **kw):
        return self.fs.fs_attention_forward(self.fmt, self.X, self.Y, self.H, scale=self.scale, bias=self.bias, dropout=self.drop, **kw)

    def backward(self, out, lse, **kw):
        return self.fs.fs_attention_backward(self.fmt, self.fmt_t, self.X, self.Y, self.H, out, lse, self.G, scale=self.scale, bias=self.bias, dropout=self.drop, **kw)

    def check(self):
        out, lse = self.forward()
        want, wl, eo, el = self.ref.forward()
        near(out, want, eo, "out")
        fine = np.isfinite(wl)
        got = self.f64(lse)
        assert np.array_equal(np.isneginf(got), ~fine)
        near(got[fine], wl[fine], el[fine], "lse")
        grads = self.backward(out, lse)
        want, bound = self.ref.backward(self.f64(out), got, self.f64(self.G))
        for k, g in zip(("dX", "dY", "dH", "dTable"), grads):
            assert (g is None) == (k not in want)
            if g is not None:
                near(g, want[k], bound[k], k)
        return out, lse, grads


def near(got, want, bound, what):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else got
    assert got.shape == want.shape, what
    worst = float((np.abs(got - want) / bound).max()) if got.size else 0.0
    print("%s: %.3f of the bound" % (what, worst), flush=True)
    assert worst <= 1.0, what


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("V,V_t,chunk", [(4, 8, 0), (8, 16, 32), (16, 4, 64), (8, 8, 0)])
@pytest.mark.parametrize("heads,kv,d,N,p,bias", [(1, 1, 32, 64, 0.0, None), (2, 1, 40, 24, 0.25, (20, 30)), (3, 3, 128, 128, 0.5, None), (6, 2, 64, 32, 0.0, (32, 128))])
def test_heads_windows_and_types(fs, dtype, V, V_t, chunk, heads, kv, d, N, p, bias):
    Problem(fs, 1, 121, 150, heads, kv, d, N, dtype, kind="hub", p=p, bias=bias, V=V, V_t=V_t, chunk=chunk).check()


@pytest.mark.parametrize("d", [8, 16, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("N", [8, 32, 48, 64, 104, 128])
def test_every_width(fs, d, N):
    Problem(fs, 2, 70, 61, 2, 1, d, N, "f16" if (d + N) % 16 else "bf16", p=0.1, bias=(7, 9)).check()


@pytest.mark.parametrize("M,K,kind", [(1, 1, "dense"), (1, 700, "dense"), (500, 1, "dense"), (7, 33, "dense"), (100, 100, "band"), (64, 300, "hub"), (40, 50, "empty"), (17, 16, "random")])
@pytest.mark.parametrize("p,bias", [(0.0, None), (0.3, (32, 1024))])
def test_shapes_from_one_token_on(fs, M, K, kind, p, bias):
    Problem(fs, 3, M, K, 4, 2, 64, 64, "bf16", kind=kind, p=p, bias=bias, shift=K - M).check()


@pytest.mark.parametrize("layout", ["heads", "wide"])
def test_strides_and_outputs_in_place_of_new_ones(fs, layout):
    import torch
    a = Problem(fs, 4, 90, 77, 4, 2, 24, 40, "f16", kind="hub", p=0.2, bias=(16, 20), layout=layout)
    out, lse, grads = a.check()
    wide = torch.full((90 + 3, 4, 56), 5.0, dtype=torch.float16, device="cuda")
    to = wide[:90, :, 8:48]
    got, _ = a.forward(out=to)
    assert torch.equal(got, out) and (wide[90:] == 5.0).all() and (wide[:, :, :8] == 5.0).all() and (wide[:, :, 48:] == 5.0).all()
    rows = torch.full((77 + 2, 2, 32), 5.0, dtype=torch.float16, device="cuda")
    got = a.backward(out, lse, dY=rows[:77, :, :24])
    assert torch.equal(got[1], grads[1]) and (rows[77:] == 5.0).all() and (rows[:, :, 24:] == 5.0).all()
    assert all(torch.equal(g, w) for g, w in zip(got, grads))


def test_two_dimensions_are_one_head(fs):
    import torch
    a = Problem(fs, 5, 60, 44, 1, 1, 32, 48, "bf16", p=0.3, bias=(12, 8))
    out, lse, grads = a.check()
    bias = fs.FsBucketBias(a.bias.table[0], a.bias.buckets)
    o, l = fs.fs_attention_forward(a.fmt, a.X[:, 0], a.Y[:, 0], a.H[:, 0], scale=a.scale, bias=bias, dropout=a.drop)
    assert torch.equal(o, out[:, 0]) and torch.equal(l, lse[0])
    g = fs.fs_attention_backward(a.fmt, a.fmt_t, a.X[:, 0], a.Y[:, 0], a.H[:, 0], o, l, a.G[:, 0], scale=a.scale, bias=bias, dropout=a.drop)
    assert all(torch.equal(x, y[:, 0] if y.dim() == 3 else y[0]) for x, y in zip(g, grads))


def test_without_bias_and_dropout_it_is_fs_attention(fs):
    """One head: the same definition as the inference call (which rounds the same, and may add in another order)."""
    a = Problem(fs, 6, 203, 150, 1, 1, 64, 64, "f16", kind="hub")
    out, _, _ = a.check()
    other = fs.fs_attention(a.fmt, a.X[:, 0], a.Y[:, 0], a.H[:, 0], scale=a.scale)
    _, _, bound, _ = a.ref.forward()
    near(other, a.f64(out)[:, 0], 2 * bound[:, 0], "fs_attention")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_bias_of_minus_infinity_takes_entries_and_rows_out(fs, dtype):
    """The bucket of everything in front of the row: entries there count as not stored, and the first rows keep nothing."""
    import torch
    a = Problem(fs, 7, 50, 50, 2, 1, 32, 32, dtype, kind="dense", p=0.2, bias=(4, 3))
    a.bias.buckets.copy_(torch.tensor([0, 1, 2, 0, 3, 3, 3], dtype=torch.uint8))
    a.bias.table[:, 3] = -np.inf  # columns behind the row
    a.bias.table[1, :3] = -np.inf  # the second head: nothing at all
    a.ref = Attention(a.stored, a.f64(a.X), a.f64(a.Y), a.f64(a.H), a.scale, a.f64(a.bias.table), a.bias.buckets.cpu().numpy(), 0, 0.2, a.state.tolist(), dtype)
    out, lse, grads = a.check()
    assert not out[:, 1].any() and torch.isneginf(lse[1]).all() and not grads[0][:, 1].any() and not grads[3][:, 3].any()


def test_rows_with_long_tails_of_small_probabilities(fs):
    """A row of 6000 entries (parts of several items) beside rows of one: fp16 keeps the probabilities of 1 / 6000 in dH."""
    M, K = 24, 6000
    a = Problem(fs, 8, M, K, 1, 1, 16, 16, "f16", kind="dense")
    a.check()


def test_buckets_past_the_table_count_as_its_last(fs):
    import torch
    a = Problem(fs, 9, 40, 40, 1, 1, 16, 16, "f16", kind="band", bias=(5, 10))
    a.bias.buckets[::3] = 250
    a.ref.bucket = bucket_of(40, 40, a.bias.buckets.cpu().numpy(), 0, 5)
    a.check()


def test_saturating_shift(fs):
    for shift in ((1 << 31) - 1, -(1 << 31) + 1):
        a = Problem(fs, 10, 30, 30, 1, 1, 16, 16, "f16", bias=(8, 5), shift=shift)
        assert len(set(a.ref.bucket.ravel().tolist())) == 1
        a.check()


def test_a_shared_table_is_one_row_for_all_heads(fs):
    import torch
    a = Problem(fs, 11, 60, 60, 4, 2, 32, 32, "bf16", bias=(9, 12))
    one = a.bias.table[:1].expand(4, 9)
    a.bias = fs.FsBucketBias(one, a.bias.buckets)
    a.ref = Attention(a.stored, a.f64(a.X), a.f64(a.Y), a.f64(a.H), a.scale, a.f64(one), a.bias.buckets.cpu().numpy(), 0, 0.0, (0, 0), "bf16")
    out, lse = a.forward()
    want, _, eo, _ = a.ref.forward()
    near(out, want, eo, "out")
    g = a.backward(out, lse, dTable=torch.empty(4, 9, dtype=torch.bfloat16, device="cuda"))
    want, bound = a.ref.backward(a.f64(out), a.f64(lse), a.f64(a.G))
    near(g[3], want["dTable"], bound["dTable"], "dTable")


def test_results_repeat_bit_for_bit_on_another_stream_and_in_a_graph(fs):
    """Training steps captured into a graph: the step is advanced inside it, so that every replay draws another mask, and each is
    compared with the eager call of that step."""
    import torch
    a = Problem(fs, 12, 150, 130, 4, 2, 64, 64, "bf16", kind="hub", p=0.3, bias=(32, 64), chunk=64)
    assert a.fmt.n_split_windows > 0 and a.fmt_t.n_split_windows > 0

    def eager(step):
        a.state[1] = step
        out, lse = a.forward()
        return (out, lse) + a.backward(out, lse)

    want = [eager(k) for k in range(4)]
    assert not torch.equal(want[0][0], want[1][0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.state[1] = 2
    side.wait_stream(torch.cuda.current_stream())
    out, lse = a.forward(stream=side)
    got = (out, lse) + a.backward(out, lse, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[2]))
    M, n = 150, 32
    bufs = [torch.empty_like(t) for t in want[0]]
    fwork = torch.empty(max(fs.fs_attention_forward_workspace_bytes(a.fmt, 4, 64), 16), dtype=torch.uint8, device="cuda")
    bwork = torch.empty(fs.fs_attention_backward_workspace_bytes(a.fmt, a.fmt_t, 4, 2, 64, 64, n), dtype=torch.uint8, device="cuda")

    def step():
        a.forward(out=bufs[0], lse=bufs[1], work=fwork)
        a.backward(bufs[0], bufs[1], dX=bufs[2], dY=bufs[3], dH=bufs[4], dTable=bufs[5], work=bwork)
        a.state[1] += 1

    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    a.state[1] = 0
    for k in range(4):
        for b in bufs:
            b.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(bufs, want[k])), k




@pytest.mark.parametrize("V", [4, 8, 16])
@pytest.mark.parametrize("p,bias", [(0.3, None), (0.0, (5, 9)), (0.3, (5, 9))])
def test_infinities_and_nan_in_rows_nobody_stores(fs, V, p, bias):
    """Rows of Y and H (backward: of X and the gradient) that a window does not reference hold no finite number, the next block's vectors
    in the arrays among them: nothing of them arrives."""
    import torch
    a = Problem(fs, 16, 64, 90, 2, 1, 32, 48, "bf16", kind="band", p=p, bias=bias, V=V, V_t=V)
    out, lse, grads = a.check()
    bad = ~a.stored.any(0)
    assert bad.any()
    rows = torch.from_numpy(np.nonzero(bad)[0]).cuda()
    a.Y[rows], a.H[rows] = float("nan"), float("inf")
    got = a.forward()
    assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    assert all(torch.equal(x, y) for x, y in zip(a.backward(out, lse), grads) if y is not None)
    # a row that only the last window references
    b = Problem(fs, 17, 64, 64, 1, 1, 32, 48, "f16", kind="random", p=p, bias=bias, V=V, V_t=V)
    stored = b.stored.copy()
    stored[:, 5] = False
    stored[-1, 5] = True
    rp, ci = csr_of(stored)
    b.fmt = fs.fs_convert(rp, ci, None, 64, 64, torch_dtype=torch.float16, V=V)
    want = b.forward()[0].clone()
    b.H[5] = float("inf")
    b.Y[5] = float("nan")
    got = b.forward()[0]
    last = (64 - 1) // V * V
    assert torch.equal(got[:last], want[:last]) and torch.isnan(got[-1]).all()


@pytest.mark.parametrize("M,K", [(0, 5), (5, 0), (0, 0)])
def test_no_rows_or_no_columns(fs, M, K):
    a = Problem(fs, 18, M, K, 2, 1, 16, 16, "f16", kind="empty", p=0.2, bias=(4, 3))
    out, lse = a.forward()
    assert out.shape == (M, 2, 16) and not out.any() and (lse == -np.inf).all()
    assert not any(g.any() for g in a.backward(out, lse))


def test_the_most_heads_for_one_of_keys_the_most_buckets_and_widths(fs):
    """64 query heads that share keys and values, 128 buckets, 1024 positions either way, 128 columns: the most LDS a call takes."""
    for V in (4, 16):
        Problem(fs, 19, 33, 40, 64, 1, 128, 128, "bf16", kind="random", p=0.2, bias=(128, 1024), V=V, V_t=V).check()


def test_two_calls_at_once_on_two_streams(fs):
    """Calls own what they write: two in flight give what they give alone."""
    import torch
    a = Problem(fs, 20, 700, 600, 2, 2, 64, 64, "f16", kind="hub", p=0.2, bias=(32, 100), chunk=64)
    b = Problem(fs, 21, 500, 800, 4, 1, 32, 32, "bf16", kind="hub", p=0.4, bias=(16, 50), chunk=64)
    want = [x.forward() + x.backward(*x.forward()) for x in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [[], []]
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                o, l = x.forward()
                got[i] = (o, l) + x.backward(o, l)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("V", [4, 8, 16])
@pytest.mark.parametrize("heads", [1, 3])
@pytest.mark.parametrize("M,K,kind", [(203, 150, "hub"), (64, 64, "band"), (1, 77, "dense"), (9, 31, "dense"), (30, 20, "empty"), (5, 1, "dense")])
def test_value_arrays(fs, dtype, V, heads, M, K, kind):
    import torch
    rng = np.random.default_rng(V + heads + M)
    stored = stored_of(rng, M, K, kind)
    rp, ci = csr_of(stored)
    fmt = fs.fs_convert(rp, ci, None, M, K, torch_dtype=torch_dtype(dtype), V=V, chunk=32)
    u, f = HALF_STEP[dtype], FLOOR[dtype]
    n = fmt.V * fmt.nvec
    slot = fmt.csr_to_slot_t().cpu().numpy()
    outside = np.ones(n, dtype=bool)
    outside[slot] = False
    vals = torch.from_numpy(rng.standard_normal((heads, n))).to(torch_dtype(dtype)).cuda()  # (something outside the pattern too)
    table = torch.from_numpy(rng.standard_normal((heads, 11))).to(torch_dtype(dtype)).cuda()
    buckets = torch.from_numpy(rng.integers(0, 11, 2 * 13 + 1).astype(np.uint8)).cuda()
    bias = fs.FsBucketBias(table, buckets, shift=3)
    bucket = bucket_of(M, K, buckets.cpu().numpy(), 3, 11)[stored]
    v = vals.double().cpu().numpy()[:, slot]
    t = table.double().cpu().numpy()[:, bucket]
    got = fs.fs_edge_bias(fmt, vals, bias, scale=-0.7).double().cpu().numpy()
    near(got[:, slot], -0.7 * v + t, u * np.abs(-0.7 * v + t) + 2.0 ** -22 * (np.abs(v) + np.abs(t)) + f, "bias")
    assert not got[:, outside].any() and not np.signbit(got[:, outside]).any()
    # the gradient of the table: sums of up to 2^10 values in fp32, one rounding
    want = np.stack([np.bincount(bucket, weights=x, minlength=11) for x in v])
    size = np.stack([np.bincount(bucket, weights=np.abs(x), minlength=11) for x in v])
    grad = fs.fs_edge_bias_backward(fmt, vals, bias)
    near(grad, want, u * np.abs(want) + 2.0 ** -13 * size + f, "dtable")
    assert torch.equal(grad, fs.fs_edge_bias_backward(fmt, vals, bias))
    # dropout: the kept ones exactly the reference's
    state = torch.tensor([(1 << 40) + 17, 5], device="cuda")
    drop = fs.FsDropout(0.37, state)
    z = keep_factors(heads, M, K, 0.37, state.tolist())[:, stored]
    got = fs.fs_edge_dropout(fmt, vals, drop).double().cpu().numpy()
    near(got[:, slot], v * z, u * np.abs(v * z) + 2.0 ** -22 * np.abs(v) + f * (z > 0) + 1e-300, "dropout")
    assert not got[:, outside].any()
    same = vals.clone()
    assert torch.equal(fs.fs_edge_dropout(fmt, same, drop, out=same).double().cpu(), torch.from_numpy(got)) and fs.fs_edge_dropout(fmt, vals, fs.FsDropout(0.0, state)).double().cpu().numpy()[:, slot].tolist() == v.tolist()
    same = vals.clone()
    fs.fs_edge_bias(fmt, same, bias, scale=-0.7, out=same)
    assert torch.equal(same, fs.fs_edge_bias(fmt, vals, bias, scale=-0.7))


def test_value_arrays_of_one_element_alignment(fs):
    """Arrays that begin on any element, with guards around them."""
    import torch
    rng = np.random.default_rng(0)
    stored = stored_of(rng, 70, 90, "random")
    rp, ci = csr_of(stored)
    for V in (4, 8, 16):
        fmt = fs.fs_convert(rp, ci, None, 70, 90, torch_dtype=torch.float16, V=V)
        n = fmt.V * fmt.nvec
        vals = torch.from_numpy(rng.standard_normal(n)).half().cuda()
        buckets = torch.zeros(3, dtype=torch.uint8, device="cuda")
        bias = fs.FsBucketBias(torch.ones(1, dtype=torch.float16, device="cuda"), buckets)
        drop = fs.FsDropout(0.5, torch.tensor([1, 2], device="cuda"))
        for call in (lambda t, o: fs.fs_edge_bias(fmt, t, bias, out=o), lambda t, o: fs.fs_edge_dropout(fmt, t, drop, out=o)):
            want = call(vals, None)
            a, b = torch.full((n + 9,), 3.0, dtype=torch.float16, device="cuda"), torch.full((n + 9,), 3.0, dtype=torch.float16, device="cuda")
            a[1:n + 1] = vals
            call(a[1:n + 1], b[3:n + 3])
            assert torch.equal(b[3:n + 3], want) and (b[:3] == 3.0).all() and (b[n + 3:] == 3.0).all()


@pytest.mark.parametrize("kind", ["sparse", "band"])
@pytest.mark.parametrize("heads,n_buckets,reach", [(1, 32, 128), (3, 128, 1024), (2, 1, 0)])
@pytest.mark.parametrize("V", [4, 8])
def test_bias_over_many_blocks(fs, kind, heads, n_buckets, reach, V):
    """More blocks than wavefronts, more of their tables than one launch adds.  Gradients of -1, 0 and 1: every sum is a whole number below
    2^24, so fp32 holds it whatever the order, and the result is the sum rounded once (whole numbers up to 2048 as they are, f16)."""
    import torch
    rng = np.random.default_rng(n_buckets + V)
    if kind == "sparse":
        M = K = 50000
        rows = np.repeat(np.arange(M), 18)
        cols = rng.integers(0, K, rows.size)
        near = rng.random(rows.size) < 0.5
        cols[near] = np.clip(rows[near] + rng.integers(-700, 700, near.sum()), 0, K - 1)
    else:
        M = K = 16000
        rows = np.repeat(np.arange(M), 190)
        cols = rows - np.tile(np.arange(190), M)
        rows, cols = rows[cols >= 0], cols[cols >= 0]
    at = np.unique(rows.astype(np.int64) * K + cols)
    rows, cols = at // K, at % K
    rp = np.concatenate([[0], np.cumsum(np.bincount(rows, minlength=M))])
    fmt = fs.fs_convert(to_dev_i32(rp), to_dev_i32(cols), None, M, K, torch_dtype=torch.float16, V=V)
    assert (2 * fmt.nnz < fmt.V * fmt.nvec) == (kind == "sparse")
    lut = rng.integers(0, n_buckets, 2 * reach + 1).astype(np.uint8)
    table = rng.standard_normal((heads, n_buckets)).astype(np.float16)
    bias = fs.FsBucketBias(torch.from_numpy(table).cuda(), torch.from_numpy(lut).cuda(), shift=3)
    bucket = lut[np.clip(cols - rows - 3, -reach, reach) + reach]
    g = rng.integers(-1, 2, (heads, rows.size)).astype(np.float16)
    vals = torch.stack([fs.fs_csr_to_blk(fmt, torch.from_numpy(x).cuda()) for x in g])
    want = np.stack([np.bincount(bucket, weights=x.astype(np.float64), minlength=n_buckets) for x in g]).astype(np.float16)
    for _ in range(2):
        assert np.array_equal(fs.fs_edge_bias_backward(fmt, vals, bias).cpu().numpy(), want)
    got = fs.fs_edge_bias(fmt, vals, bias, scale=0.0)
    for h in range(heads):
        assert np.array_equal(fs.fs_blk_to_csr(fmt, got[h]).cpu().numpy(), table[h][bucket])


def test_the_separate_calls_are_the_fused_one(fs):
    """SDDMM, bias, softmax, dropout, SpMM, and back: the same numbers up to the roundings in between."""
    import torch
    a = Problem(fs, 13, 180, 160, 1, 1, 32, 64, "bf16", kind="hub", p=0.3, bias=(32, 40))
    X, Y, H, G, fmt, fmt_t = a.X[:, 0], a.Y[:, 0], a.H[:, 0].contiguous(), a.G[:, 0], a.fmt, a.fmt_t
    s = fs.fs_edge_bias(fmt, fs.fs_sddmm(fmt, X, Y), fs.FsBucketBias(a.bias.table[0], a.bias.buckets), scale=a.scale)
    P = fs.fs_edge_softmax(fmt, s)
    W = fs.fs_edge_dropout(fmt, P, a.drop)
    out = fs.fs_spmm(fmt, H, vals=W)
    dS = fs.fs_edge_softmax_backward(fmt, P, fs.fs_edge_dropout(fmt, fs.fs_sddmm(fmt, G, H), a.drop))
    dT = fs.fs_edge_bias_backward(fmt, dS, fs.FsBucketBias(a.bias.table[0], a.bias.buckets))
    dX = fs.fs_spmm(fmt, Y, vals=dS).float() * a.scale
    o, l = a.forward()
    g = a.backward(o, l)

    def off(x, y):
        return ((x.float() - y.float()).norm() / y.float().norm()).item()

    # five 16-bit roundings on the way, each of 2^-8 at most, beside the fused call's two
    assert off(out, o[:, 0]) < 0.03 and off(dX, g[0][:, 0]) < 0.03 and off(dT, g[3][0]) < 0.06


def test_large_offsets_beyond_two_gibibytes(fs):
    """Rows whose byte offset passes 2^31: a wide pitch on few rows that are touched."""
    import torch
    rng = np.random.default_rng(1)
    M, K, pitch = 4, 2200, 500000  # 2200 * 1 000 000 bytes
    stored = np.zeros((M, K), dtype=bool)
    stored[:, [0, 1, 5, 2150, 2199]] = True
    rp, ci = csr_of(stored)
    fmt = fs.fs_convert(rp, ci, None, M, K, torch_dtype=torch.float16)
    rpt, cit, _ = fs.fs_csr_transpose(rp, ci, M, K)
    fmt_t = fs.fs_convert(rpt, cit, None, K, M, torch_dtype=torch.float16)
    store = torch.empty((K, pitch), dtype=torch.float16, device="cuda")
    Y, H = store[:, 8:24], store[:, 64:80]
    Y.copy_(torch.from_numpy(rng.standard_normal((K, 16))))
    H.copy_(torch.from_numpy(rng.standard_normal((K, 16))))
    X, G = (torch.from_numpy(rng.standard_normal((M, 16))).half().cuda() for _ in range(2))
    o, l = fs.fs_attention_forward(fmt, X, Y, H)
    o2, l2 = fs.fs_attention_forward(fmt, X, Y.contiguous(), H.contiguous())
    assert torch.equal(o, o2) and torch.equal(l, l2)
    dY, dH = store[:, 128:144], store[:, 256:272]
    a = fs.fs_attention_backward(fmt, fmt_t, X, Y, H, o, l, G, dY=dY, dH=dH)
    b = fs.fs_attention_backward(fmt, fmt_t, X, Y.contiguous(), H.contiguous(), o, l, G)
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


def test_refusals(fs):
    """Every refusal comes before a launch: outputs keep what they held."""
    import torch
    from paper_2412_11007_amd.binding import _FsBucketBiasStruct, _FsDropoutStruct, _FsHeadMatrix
    a = Problem(fs, 14, 40, 30, 2, 1, 16, 24, "f16", kind="hub", p=0.2, bias=(8, 6), chunk=32)
    lib = fs.load_library()
    out = torch.full((40, 2, 24), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.empty(2, 40, device="cuda")
    need = max(fs.fs_attention_forward_workspace_bytes(a.fmt, 2, 24), 16)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(heads=2, kv=1, d=16, N=24, scale=1.0, X={}, Y={}, H={}, O={}, bias={}, drop={}, work_bytes=need, fmt=a.fmt):
        def m(t, change):
            s = _FsHeadMatrix(t.data_ptr(), t.stride(0), t.stride(1))
            for k, v in change.items():
                setattr(s, k, v)
            return ctypes.byref(s)
        b = _FsBucketBiasStruct(a.bias.table.data_ptr(), 8, a.bias.buckets.data_ptr(), 8, 6, 0)
        dr = _FsDropoutStruct(0.2, a.state.data_ptr())
        for k, v in bias.items():
            setattr(b, k, v)
        for k, v in drop.items():
            setattr(dr, k, v)
        return lib.fs_attention_forward(ctypes.byref(fmt.c), heads, kv, d, N, scale, m(a.X, X), m(a.Y, Y), m(a.H, H), ctypes.byref(b), ctypes.byref(dr), m(out, O),
                                        lse.data_ptr(), work.data_ptr(), work_bytes, None)

    X = a.X.data_ptr()
    for code, kw in [(1, dict(heads=0)), (1, dict(kv=0)), (1, dict(heads=3, kv=2)), (1, dict(d=12)), (1, dict(N=20)), (1, dict(d=0)), (3, dict(d=136, X=dict(ld=272))),
                     (1, dict(scale=float("nan"))), (1, dict(scale=float("inf"))), (1, dict(X=dict(d=None))), (1, dict(X=dict(d=X + 2))), (1, dict(X=dict(ld=8))),
                     (1, dict(X=dict(ld=36))), (1, dict(X=dict(head=12))), (1, dict(X=dict(head=-16))), (1, dict(O=dict(head=16))), (3, dict(X=dict(ld=1 << 24))),
                     (1, dict(bias=dict(n_buckets=0))), (3, dict(bias=dict(n_buckets=129, ld=129))), (3, dict(bias=dict(reach=1025))), (1, dict(bias=dict(reach=-1))),
                     (1, dict(bias=dict(d_table=None))), (1, dict(bias=dict(d_bucket=None))), (1, dict(bias=dict(d_bucket=a.bias.buckets.data_ptr() + 1))),
                     (1, dict(bias=dict(ld=7))), (1, dict(bias=dict(shift=1 << 31))), (1, dict(drop=dict(p=1.0))), (1, dict(drop=dict(p=-0.1))),
                     (1, dict(drop=dict(p=float("nan")))), (1, dict(drop=dict(d_state=None)))]:
        assert call(**kw) == code, kw
    if fs.fs_attention_forward_workspace_bytes(a.fmt, 2, 24):
        assert call(work_bytes=need - 4) == 4
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    assert call() == 0
    # the backward call: another matrix's transpose, no room, an output whose heads overlap
    o, l = a.forward()
    other = Problem(fs, 15, 30, 40, 1, 1, 16, 24, "f16")
    with pytest.raises(fs.FsError) as e:
        fs.fs_attention_backward(a.fmt, a.fmt, a.X, a.Y, a.H, o, l, a.G)
    assert e.value.code == 1
    with pytest.raises(fs.FsError) as e:
        fs.fs_attention_backward(a.fmt, other.fmt, a.X, a.Y, a.H, o, l, a.G)
    assert e.value.code == 1
    with pytest.raises(fs.FsError) as e:
        fs.fs_attention_backward(a.fmt, a.fmt_t, a.X, a.Y, a.H, o, l, a.G, work=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 4
    with pytest.raises(fs.FsError) as e:
        fs.fs_attention_backward(a.fmt, a.fmt_t, a.X, a.Y, a.H, o, l, a.G, dX=torch.empty(40, 1, 16, dtype=torch.float16, device="cuda").expand(40, 2, 16))
    assert e.value.code == 1
    vals = torch.zeros(2, a.fmt.V * a.fmt.nvec, dtype=torch.float16, device="cuda")
    for bad in (lambda: fs.fs_edge_bias(a.fmt, vals, a.bias, scale=float("nan")), lambda: fs.fs_edge_dropout(a.fmt, vals, fs.FsDropout(1.0, a.state))):
        with pytest.raises(fs.FsError) as e:
            bad()
        assert e.value.code == 1
    for bad in (lambda: fs.fs_edge_bias(a.fmt, vals[0], a.bias), lambda: fs.fs_edge_dropout(a.fmt, vals[:, 1:], a.drop), lambda: fs.fs_edge_dropout(a.fmt, vals.float(), a.drop),
                lambda: fs.FsDropout(0.1, a.state.int()), lambda: fs.FsBucketBias(a.bias.table, a.bias.buckets[1:])):
        with pytest.raises(AssertionError):
            bad()


def test_outputs_and_workspaces_elsewhere_are_refused(fs):
    """Memory of the host, or a workspace with gaps, never becomes a kernel's argument."""
    import torch
    a = Problem(fs, 5, 40, 30, 2, 2, 16, 24, "f16", p=0.2, bias=(8, 5))
    o, l = a.forward()
    vals = torch.zeros(2, a.fmt.V * a.fmt.nvec, dtype=torch.float16, device="cuda")
    gaps = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[::2]
    host = torch.empty(1 << 20, dtype=torch.uint8)
    run = dict(scale=a.scale, bias=a.bias, dropout=a.drop)
    calls = [lambda: fs.fs_edge_bias(a.fmt, vals, a.bias, out=vals.cpu()), lambda: fs.fs_edge_dropout(a.fmt, vals, a.drop, out=vals.cpu()),
             lambda: fs.fs_edge_bias_backward(a.fmt, vals, a.bias, out=a.bias.table.cpu()),
             lambda: fs.fs_attention_forward(a.fmt, a.X, a.Y, a.H, out=o.cpu(), **run), lambda: fs.fs_attention_forward(a.fmt, a.X, a.Y, a.H, lse=l.cpu(), **run),
             lambda: fs.fs_attention_forward(a.fmt, a.X, a.Y.cpu(), a.H, **run),
             lambda: fs.fs_attention_backward(a.fmt, a.fmt_t, a.X, a.Y, a.H, o, l.cpu(), a.G, **run),
             lambda: fs.fs_attention_backward(a.fmt, a.fmt_t, a.X, a.Y, a.H, o, l, a.G, dTable=a.bias.table.cpu(), **run)]
    for work in (gaps, host):
        calls += [lambda work=work: fs.fs_edge_bias_backward(a.fmt, vals, a.bias, work=work),
                  lambda work=work: fs.fs_attention_forward(a.fmt, a.X, a.Y, a.H, work=work, **run),
                  lambda work=work: fs.fs_attention_backward(a.fmt, a.fmt_t, a.X, a.Y, a.H, o, l, a.G, work=work, **run)]
    for call in calls:
        with pytest.raises(AssertionError):
            call()


def test_sums_of_many_wavefronts_stay_in_the_workspace(fs):
    """128 buckets and more than 16384 items: the sums go through two launches.  What lies behind the workspace is left alone."""
    import torch
    rng = np.random.default_rng(9)
    M, deg = 120000, 6
    cols = np.sort((np.arange(M)[:, None] * 7 + np.cumsum(rng.integers(1, 9000, (M, deg)), axis=1)) % M, axis=1)
    at = np.unique(np.arange(M)[:, None] * M + cols)
    rows, cols = at // M, at % M
    rp = to_dev_i32(np.concatenate([[0], np.cumsum(np.bincount(rows, minlength=M))]))
    ci = to_dev_i32(cols)
    fmt = fs.fs_convert(rp, ci, None, M, M, torch_dtype=torch.float16, V=4, chunk=32)
    rpt, cit, _ = fs.fs_csr_transpose(rp, ci, M, M)
    fmt_t = fs.fs_convert(rpt, cit, None, M, M, torch_dtype=torch.float16, V=4)
    assert fmt.n_items > 16384
    X, Y, H, G = (torch.from_numpy(rng.standard_normal((M, 1, 8))).half().cuda() for _ in range(4))
    lut = torch.from_numpy((np.arange(2049) % 128).astype(np.uint8)).cuda()
    bias = fs.FsBucketBias(torch.from_numpy(rng.standard_normal((1, 128))).half().cuda(), lut)
    o, l = fs.fs_attention_forward(fmt, X, Y, H, scale=0.3, bias=bias)
    want = fs.fs_attention_backward(fmt, fmt_t, X, Y, H, o, l, G, scale=0.3, bias=bias)
    need = fs.fs_attention_backward_workspace_bytes(fmt, fmt_t, 1, 1, 8, 8, 128)
    store = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
    got = fs.fs_attention_backward(fmt, fmt_t, X, Y, H, o, l, G, scale=0.3, bias=bias, work=store[:need])
    assert bool((store[need:] == 0xA5).all()) and all(torch.equal(a, b) for a, b in zip(got, want))
