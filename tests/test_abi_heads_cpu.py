"""The calls with heads, biases and dropout as far as the host goes: layouts of their structs, workspace sizes, and refusals, all of
which come before anything is launched."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def fs():
    import paper_2412_11007_amd as fs
    if not os.path.exists(fs.library_path()):
        from paper_2412_11007_amd.build import build_library
        build_library()
    fs.load_library()
    return fs


def test_struct_layouts(fs, tmp_path):
    from paper_2412_11007_amd import binding
    structs = {"fs_bucket_bias": binding._FsBucketBiasStruct, "fs_dropout": binding._FsDropoutStruct, "fs_head_matrix": binding._FsHeadMatrix}
    prog = "#include <stdio.h>\n#include <stddef.h>\n#include \"flashsparse.h\"\nint main(void){\n"
    for c, s in structs.items():
        prog += "printf(\"%%zu\\n\", sizeof(%s));\n" % c
        for f in s._fields_:
            prog += "printf(\"%%zu\\n\", offsetof(%s, %s));\n" % (c, f[0])
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text(prog + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = iter(subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    for s in structs.values():
        assert int(next(got)) == ctypes.sizeof(s)
        for f in s._fields_:
            assert int(next(got)) == getattr(s, f[0]).offset


class Call:
    """A call that would be valid (on made-up addresses) but for what a test changes: no such call gets as far as a launch."""

    def __init__(self, fs):
        from paper_2412_11007_amd import binding as b
        self.b, self.lib = b, fs.load_library()
        self.fmt, self.fmt_t = self.format(b, 100, 80), self.format(b, 80, 100)

    @staticmethod
    def format(b, M, K):
        f = b._FsFormatStruct()
        f.M, f.K, f.nnz, f.nvec, f.W, f.V, f.KB, f.dtype, f.chunk = M, K, 500, 400, (M + 7) // 8, 8, 32, 0, 256
        f.n_items, f.n_split_items, f.n_split_windows, f.n_blocks, f.n_cut_items = 13, 4, 1, 20, 4
        for name in ("win_ptr", "vec_col", "vec_mask", "csr_to_slot", "vals_blk", "blk_desc", "items", "split_windows", "item_order", "items_by_cost",
                     "blk_row_base", "slot_range", "blk_row_bits"):
            setattr(f, name, 0x1000)
        return f

    def matrix(self, heads, columns, **kw):
        m = self.b._FsHeadMatrix(0x100000, heads * columns, columns)
        for k, v in kw.items():
            setattr(m, k, v)
        return ctypes.byref(m)

    def bias(self, **kw):
        s = self.b._FsBucketBiasStruct(0x2000, 8, 0x3000, 8, 6, 0)
        for k, v in kw.items():
            setattr(s, k, v)
        return ctypes.byref(s)

    def drop(self, **kw):
        s = self.b._FsDropoutStruct(0.5, 0x4000)
        for k, v in kw.items():
            setattr(s, k, v)
        return ctypes.byref(s)

    def forward(self, heads=4, kv=2, d=16, N=24, scale=1.0, X={}, Y={}, H={}, O={}, bias={}, drop={}, lse=0x5000, work=0x10000, work_bytes=0, fmt={}):
        f = self.format(self.b, 100, 80)
        for k, v in fmt.items():
            setattr(f, k, v)
        return self.lib.fs_attention_forward(ctypes.byref(f), heads, kv, d, N, scale, self.matrix(4, 16, **X), self.matrix(2, 16, **Y), self.matrix(2, 24, **H),
                                             self.bias(**bias), self.drop(**drop), self.matrix(4, 24, **O), lse, work, work_bytes, None)

    def backward(self, heads=4, kv=2, d=16, N=24, G={}, dX={}, dY={}, dH={}, lse=0x5000, grad=0x6000, work=0x10000, work_bytes=0, fmt_t={}, with_bias=True):
        t = self.format(self.b, 80, 100)
        for k, v in fmt_t.items():
            setattr(t, k, v)
        return self.lib.fs_attention_backward(ctypes.byref(self.fmt), ctypes.byref(t), heads, kv, d, N, 1.0, self.matrix(4, 16), self.matrix(2, 16), self.matrix(2, 24),
                                              self.bias() if with_bias else None, self.drop(), self.matrix(4, 24), lse, self.matrix(4, 24, **G), self.matrix(4, 16, **dX),
                                              self.matrix(2, 16, **dY), self.matrix(2, 24, **dH), grad, work, work_bytes, None)


FORWARD = [
    (1, dict(heads=0)), (1, dict(heads=-4)), (1, dict(kv=0)), (1, dict(heads=3)), (1, dict(d=12)), (1, dict(d=0)), (1, dict(N=20)), (1, dict(N=0)), (3, dict(d=136)),
    (3, dict(N=136)), (3, dict(heads=65536, kv=65536)), (3, dict(heads=130, kv=2)), (1, dict(scale=float("nan"))), (1, dict(scale=float("-inf"))),
    (1, dict(X=dict(d=None))), (1, dict(Y=dict(d=0x100008))), (1, dict(H=dict(ld=16))), (1, dict(X=dict(ld=60))), (1, dict(X=dict(head=4))), (1, dict(Y=dict(head=-16))),
    (1, dict(O=dict(head=16))), (3, dict(X=dict(ld=1 << 23))), (3, dict(Y=dict(head=1 << 46))), (1, dict(bias=dict(n_buckets=0))), (1, dict(bias=dict(reach=-1))),
    (3, dict(bias=dict(n_buckets=129, ld=129))), (3, dict(bias=dict(reach=1025))), (1, dict(bias=dict(d_table=None))), (1, dict(bias=dict(d_table=0x2001))),
    (1, dict(bias=dict(d_bucket=None))), (1, dict(bias=dict(d_bucket=0x3002))), (1, dict(bias=dict(ld=7))), (1, dict(bias=dict(ld=-8))),
    (1, dict(bias=dict(shift=1 << 31))), (1, dict(bias=dict(shift=-(1 << 31)))), (1, dict(drop=dict(p=1.0))), (1, dict(drop=dict(p=-0.001))),
    (1, dict(drop=dict(p=float("nan")))), (1, dict(drop=dict(d_state=None))), (1, dict(drop=dict(d_state=0x4004))), (1, dict(lse=0x5002)), (1, dict(work=None)),
    (1, dict(work=0x10008)), (4, dict()), (4, dict(work_bytes=4 * 4 * 8 * 26 * 4 - 1)), (3, dict(fmt=dict(V=2))), (3, dict(fmt=dict(KB=64))),
    (1, dict(fmt=dict(blk_row_bits=None))), (3, dict(fmt=dict(M=1 << 24))), (1, dict(fmt=dict(n_items=-1)))]


@pytest.mark.parametrize("code,change", FORWARD)
def test_forward_refuses(fs, code, change):
    assert Call(fs).forward(**change) == code


BACKWARD = [
    (1, dict(fmt_t=dict(M=81))), (1, dict(fmt_t=dict(K=99))), (1, dict(fmt_t=dict(nnz=499))), (1, dict(fmt_t=dict(dtype=1))), (1, dict(fmt_t=dict(blk_row_bits=None))),
    (3, dict(fmt_t=dict(V=32))), (1, dict(G=dict(d=None))), (1, dict(dX=dict(d=None))), (1, dict(dY=dict(ld=8))), (1, dict(dH=dict(head=16))), (1, dict(dX=dict(head=0))),
    (1, dict(lse=None)), (1, dict(grad=0x6001)), (1, dict(with_bias=False)), (1, dict(work=None)), (4, dict())]


@pytest.mark.parametrize("code,change", BACKWARD)
def test_backward_refuses(fs, code, change):
    assert Call(fs).backward(**change) == code


def test_value_array_calls_refuse(fs):
    c = Call(fs)
    f = ctypes.byref(c.fmt)

    def bias(heads=2, vals=0x8000, scale=1.0, b={}, out=0x9000):
        return c.lib.fs_edge_bias(f, heads, vals, scale, c.bias(**b), out, None)

    for code, kw in [(1, dict(heads=-1)), (3, dict(heads=65536)), (1, dict(vals=None)), (1, dict(vals=0x8001)), (1, dict(out=None)), (1, dict(out=0x9001)),
                     (1, dict(scale=float("inf"))), (1, dict(b=dict(ld=3))), (3, dict(b=dict(reach=2000))), (0, dict(heads=0))]:
        assert bias(**kw) == code, kw
    assert c.lib.fs_edge_bias(f, 1, 0x8000, 1.0, None, 0x9000, None) == 1
    assert c.lib.fs_edge_dropout(f, 1, 0x8000, None, 0x9000, None) == 1
    assert c.lib.fs_edge_dropout(f, 1, 0x8000, c.drop(p=1.5), 0x9000, None) == 1
    assert c.lib.fs_edge_dropout(f, 1, None, c.drop(), 0x9000, None) == 1
    n = ctypes.c_size_t(0)
    assert c.lib.fs_edge_bias_backward_workspace_bytes(f, 2, 8, ctypes.byref(n)) == 0 and n.value > 0
    assert c.lib.fs_edge_bias_backward_workspace_bytes(f, 2, 129, ctypes.byref(n)) == 3
    assert c.lib.fs_edge_bias_backward_workspace_bytes(f, 2, 8, None) == 1
    for code, args in [(1, (None, 0xA000, 0x10000, 1 << 20)), (1, (0x8000, None, 0x10000, 1 << 20)), (1, (0x8000, 0xA001, 0x10000, 1 << 20)), (1, (0x8000, 0xA000, None, 1 << 20)),
                       (4, (0x8000, 0xA000, 0x10000, 64))]:
        assert c.lib.fs_edge_bias_backward(f, 2, args[0], c.bias(), args[1], args[2], args[3], None) == code, args


def test_workspace_sizes(fs):
    c = Call(fs)
    n = ctypes.c_size_t(0)
    f, t = ctypes.byref(c.fmt), ctypes.byref(c.fmt_t)
    # fp32 tiles of four parts of eight rows, and two statistics a row
    assert c.lib.fs_attention_forward_workspace_bytes(f, 4, 24, ctypes.byref(n)) == 0 and n.value == 4 * 4 * 8 * 26 * 4
    assert c.lib.fs_attention_forward_workspace_bytes(f, 0, 24, ctypes.byref(n)) == 1
    assert c.lib.fs_attention_backward_workspace_bytes(f, t, 4, 2, 16, 24, 0, ctypes.byref(n)) == 0
    without = n.value
    assert without >= 4 * (2 * 4 * 100 + 4 * 8 * (4 * 16 + 2 * 40))
    assert c.lib.fs_attention_backward_workspace_bytes(f, t, 4, 2, 16, 24, 8, ctypes.byref(n)) == 0
    assert n.value >= without + 4 * 4 * 13 * 8
    assert c.lib.fs_attention_backward_workspace_bytes(f, None, 4, 2, 16, 24, 0, ctypes.byref(n)) == 1


@pytest.mark.parametrize("items", [1, 33, 5000, 16385, 40000])
@pytest.mark.parametrize("buckets", [1, 32, 65, 128])
def test_workspace_holds_every_launch_of_the_sums(fs, items, buckets):
    """The wavefronts' sums, up to 1024 groups of them, and the 64 partial tables that two launches add those through."""
    c = Call(fs)
    n = ctypes.c_size_t(0)
    c.fmt.n_items = items
    f, t = ctypes.byref(c.fmt), ctypes.byref(c.fmt_t)
    assert c.lib.fs_attention_backward_workspace_bytes(f, t, 4, 2, 16, 24, 0, ctypes.byref(n)) == 0
    without = n.value
    assert c.lib.fs_attention_backward_workspace_bytes(f, t, 4, 2, 16, 24, buckets, ctypes.byref(n)) == 0
    assert n.value >= without + 4 * 4 * buckets * (items + min(1024, -(-items // 32)) + 64)
