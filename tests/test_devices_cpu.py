"""Calls whose tensors lie on different GPUs are refused.  The tensors here are fake: they have a shape, a type and a device, but no memory, so that
a machine without any GPU can have two.  A call that is not refused fails when it asks for memory."""
import os

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")  # (of one that the call then finds no memory for)

M, K, NVEC, NNZ, V = 100, 80, 400, 500, 8


@pytest.fixture(scope="module")
def fs():
    import paper_2412_11007_amd as fs
    if not os.path.exists(fs.library_path()):
        from paper_2412_11007_amd.build import build_library
        build_library()
    fs.load_library()
    return fs


def fake(*shape, gpu=0, dtype=torch.float16):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device="cuda:%d" % gpu)


def formats(fs, gpu=0, gpu_t=0):
    from paper_2412_11007_amd import binding
    out = []
    for rows, cols, g in ((M, K, gpu), (K, M, gpu_t)):
        c = binding._FsFormatStruct()
        c.M, c.K, c.nnz, c.nvec, c.V, c.dtype = rows, cols, NNZ, NVEC, V, 0
        out.append(fs.FsFormat(c, fake(64, gpu=g, dtype=torch.uint8), torch.float16))
    return out


OLD = {"spmm": (("B", (K, 16)), ("vals", (V * NVEC,))), "sddmm": (("X", (M, 16)), ("Y", (K, 16))), "softmax": (("vals", (V * NVEC,)),),
       "softmax_backward": (("probs", (V * NVEC,)), ("grad", (V * NVEC,))), "attention": (("X", (M, 16)), ("Y", (K, 16)), ("H", (K, 24))),
       "sddmm_spmm": (("X", (M, 16)), ("Y", (K, 16)), ("H", (K, 24))), "blk_to_csr": (("blk", (V * NVEC,)),), "csr_to_blk": (("vals_csr", (NNZ,)),)}
NAMES = {"softmax": "fs_edge_softmax", "softmax_backward": "fs_edge_softmax_backward"}


@pytest.fixture
def no_gpu_needed(monkeypatch):
    from paper_2412_11007_amd import binding
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)


def not_refused(call):
    """All on one device: the call gets as far as the memory."""
    with pytest.raises(RuntimeError):
        call()


def refused(call):
    with pytest.raises(AssertionError):
        call()


@pytest.mark.parametrize("name", OLD)
def test_calls_of_one_head(fs, no_gpu_needed, name):
    fmt, _ = formats(fs)
    call = getattr(fs, NAMES.get(name, "fs_" + name))
    here = {k: fake(*shape) for k, shape in OLD[name]}
    not_refused(lambda: call(fmt, **here))
    for k, shape in OLD[name]:
        refused(lambda: call(fmt, **{**here, k: fake(*shape, gpu=1)}))
    refused(lambda: call(formats(fs, gpu=1)[0], **here))


def heads_arguments(fs):
    t = dict(X=fake(M, 4, 16), Y=fake(K, 2, 16), H=fake(K, 2, 24), table=fake(4, 9), buckets=fake(7, dtype=torch.uint8), state=fake(2, dtype=torch.int64))
    u = dict(out=fake(M, 4, 24), lse=fake(4, M, dtype=torch.float32), grad=fake(M, 4, 24))
    return t, u


def split(fs, a):
    a = dict(a)
    return dict(bias=fs.FsBucketBias(a.pop("table"), a.pop("buckets")), dropout=fs.FsDropout(0.5, a.pop("state")), **a)


def elsewhere(t):
    return fake(*t.shape, gpu=1, dtype=t.dtype)


@pytest.mark.parametrize("given", [False, True])
def test_forward(fs, no_gpu_needed, given):
    fmt, _ = formats(fs)
    here, more = heads_arguments(fs)
    out = dict(out=more["out"], lse=more["lse"]) if given else {}
    not_refused(lambda: fs.fs_attention_forward(fmt, **split(fs, here), **out))
    for k in here:
        refused(lambda: fs.fs_attention_forward(fmt, **split(fs, {**here, k: elsewhere(here[k])}), **out))
    for k in out:
        refused(lambda: fs.fs_attention_forward(fmt, **split(fs, here), **{**out, k: elsewhere(out[k])}))
    refused(lambda: fs.fs_attention_forward(formats(fs, gpu=1)[0], **split(fs, here), **out))


@pytest.mark.parametrize("given", [False, True])
def test_backward(fs, no_gpu_needed, given):
    fmt, fmt_t = formats(fs)
    here, more = heads_arguments(fs)
    here.update(more)
    to = dict(dX=fake(M, 4, 16), dY=fake(K, 2, 16), dH=fake(K, 2, 24), dTable=fake(4, 9)) if given else {}
    not_refused(lambda: fs.fs_attention_backward(fmt, fmt_t, **split(fs, here), **to))
    for k in here:
        refused(lambda: fs.fs_attention_backward(fmt, fmt_t, **split(fs, {**here, k: elsewhere(here[k])}), **to))
    for k in to:
        refused(lambda: fs.fs_attention_backward(fmt, fmt_t, **split(fs, here), **{**to, k: elsewhere(to[k])}))
    refused(lambda: fs.fs_attention_backward(fmt, formats(fs, gpu_t=1)[1], **split(fs, here), **to))


def test_value_arrays(fs, no_gpu_needed):
    fmt, _ = formats(fs)
    t = dict(table=fake(2, 9), buckets=fake(7, dtype=torch.uint8), state=fake(2, dtype=torch.int64), vals=fake(2, V * NVEC))
    calls = {"fs_edge_bias": ("vals", "table", "buckets"), "fs_edge_bias_backward": ("vals", "table", "buckets"), "fs_edge_dropout": ("vals", "state")}
    for name, uses in calls.items():
        def call(a):
            return getattr(fs, name)(fmt, a["vals"], fs.FsDropout(0.5, a["state"]) if "state" in uses else fs.FsBucketBias(a["table"], a["buckets"]))
        not_refused(lambda: call(t))
        for k in uses:
            refused(lambda: call({**t, k: elsewhere(t[k])}))


def test_calls_with_heads_run_on_the_current_device(fs, no_gpu_needed, monkeypatch):
    from paper_2412_11007_amd import binding
    fmt, fmt_t = formats(fs)
    here, more = heads_arguments(fs)
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    refused(lambda: fs.fs_attention_forward(fmt, **split(fs, here)))
    refused(lambda: fs.fs_attention_backward(fmt, fmt_t, **split(fs, {**here, **more})))
    refused(lambda: fs.fs_edge_dropout(fmt, fake(2, V * NVEC), fs.FsDropout(0.5, here["state"])))
    refused(lambda: fs.fs_edge_bias(fmt, fake(4, V * NVEC), split(fs, here)["bias"]))
    refused(lambda: fs.fs_edge_bias_backward(fmt, fake(4, V * NVEC), split(fs, here)["bias"]))


def test_conversion_and_gather(fs, no_gpu_needed):
    i = lambda n, gpu=0: fake(n, gpu=gpu, dtype=torch.int32)  # noqa: E731
    refused(lambda: fs.fs_convert(i(M + 1), i(NNZ, 1), None, M, K))
    refused(lambda: fs.fs_convert(i(M + 1), i(NNZ), fake(NNZ, gpu=1), M, K))
    refused(lambda: fs.fs_csr_transpose(i(M + 1), i(NNZ, 1), M, K))
    refused(lambda: fs.fs_gather16(fake(10), i(10, 1)))
