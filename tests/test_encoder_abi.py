"""What the history encoder's entry points refuse, and the layout of their records: no GPU in it.  A refusal comes before
anything but the context's error text is touched, so a zeroed block of memory stands in for a context here."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2604_24073_amd as fs

ROOT = os.path.join(os.path.dirname(fs.LIB_PATH), "..")
P = 4096                                       # an address that is aligned and never followed


@pytest.fixture
def blank():
    return ctypes.create_string_buffer(1 << 16)


def refused(rc, want=fs.FS_EINVAL):
    assert rc == want, rc


def error(blank):
    return fs.load_library().fs_last_error(ctypes.addressof(blank)).decode()


@pytest.mark.parametrize("record", ["fs_block_args", "fs_attention_args"])
def test_records_match_a_c_compiler(tmp_path, record):
    mirror = getattr(fs, record)
    fields = [f[0] for f in mirror._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "freescale_encoder.h"\nint main(void) {\n'
                   f'  printf("%zu\\n", sizeof({record}));\n' +
                   "".join(f'  printf("%zu\\n", offsetof({record}, {n}));\n' for n in fields) + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [ctypes.sizeof(mirror)] + [getattr(mirror, n).offset for n in fields]


def block(**changes):
    rec = fs.fs_block_args(n=10, dim=64, rows_dt=fs.FS_F32, dt=fs.FS_BF16, eps=1e-6, a_stride=64, g_stride=64, da_stride=64,
                           dg_stride=64, work_bytes=1 << 20)
    for name in ("x", "a", "g", "w_post", "scale", "w_pre", "y", "h", "dy", "dh", "dx", "da", "dg", "dw_post", "dscale", "dw_pre",
                 "work"):
        setattr(rec, name, P)
    for k, v in changes.items():
        setattr(rec, k, v)
    return rec


BOTH = [dict(n=-1), dict(n=1 << 31), dict(dim=0), dict(dim=-8), dict(dim=63), dict(dim=68), dict(dim=1032), dict(rows_dt=2),
        dict(dt=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(g=None), dict(w_post=None),
        dict(scale=None), dict(w_pre=None), dict(a=P + 8), dict(g=P + 2), dict(a_stride=56), dict(g_stride=68), dict(a_stride=-64),
        dict(y=P + 4), dict(w_pre=P + 4), dict(scale=P + 8)]


@pytest.mark.parametrize("changes", BOTH + [dict(x=None), dict(x=P + 4), dict(y=None), dict(h=P + 8), dict(a=None, h=None),
                                            dict(a_codes=P), dict(y_codes=P), dict(g_codes=P + 8, g_exps=P),
                                            dict(a_codes=P, a_exps=P, dim=40, a_stride=40, g_stride=40)])
def test_block_norm_refuses(blank, changes):
    rec = block(**changes)
    refused(fs.load_library().fs_block_norm(ctypes.addressof(blank), ctypes.byref(rec), None))
    assert "block norm" in error(blank)


@pytest.mark.parametrize("changes", BOTH + [dict(y=None), dict(dx=None), dict(dx=P + 4), dict(dy=P + 4), dict(da=None), dict(dg=None),
                                            dict(da=P + 8), dict(da_stride=56), dict(dg_stride=60), dict(dw_post=None),
                                            dict(dscale=None), dict(dw_pre=None), dict(work=None), dict(work_bytes=8),
                                            dict(a=None, dh=None), dict(a=None, a_codes=P), dict(g=None, g_codes=P),
                                            dict(y=None, y_codes=P), dict(a=None, a_codes=P, a_exps=P, dim=40),
                                            dict(dh=P + 2)])
def test_block_norm_backward_refuses(blank, changes):
    rec = block(**changes)
    refused(fs.load_library().fs_block_norm_backward(ctypes.addressof(blank), ctypes.byref(rec), None))
    assert "block norm" in error(blank)


def test_null_records_and_contexts(blank):
    lib = fs.load_library()
    for call in (lib.fs_block_norm, lib.fs_block_norm_backward):
        refused(call(None, None, None))
        refused(call(ctypes.addressof(blank), None, None))
    refused(lib.fs_rows_pack8(None, P, 32, fs.FS_F32, 1, 32, P, P, None))
    refused(lib.fs_rows_unpack8(None, P, P, 1, 32, P, 32, fs.FS_F32, None))


def test_no_rows_are_no_work(blank):
    lib, ctx = fs.load_library(), ctypes.addressof(blank)
    assert lib.fs_block_norm(ctx, ctypes.byref(block(n=0)), None) == fs.FS_OK
    assert lib.fs_rows_pack8(ctx, None, 32, fs.FS_F32, 0, 32, None, None, None) == fs.FS_OK
    assert lib.fs_rows_unpack8(ctx, None, None, 0, 32, None, 32, fs.FS_F32, None) == fs.FS_OK
    assert lib.fs_block_norm_work_bytes(0, 64) == 0


@pytest.mark.parametrize("rows,stride,dt,n,dim,codes,exps", [
    (None, 32, 0, 1, 32, P, P), (P, 32, 0, 1, 32, None, P), (P, 32, 0, 1, 32, P, None), (P, 32, 2, 1, 32, P, P),
    (P, 32, 0, -1, 32, P, P), (P, 32, 0, 1 << 31, 32, P, P), (P, 40, 0, 1, 40, P, P), (P, 31, 0, 1, 32, P, P),
    (P, 33, 0, 1, 32, P, P), (P, 36, 1, 1, 32, P, P), (P + 4, 32, 0, 1, 32, P, P), (P, 32, 0, 1, 32, P + 8, P),
    (P, 1056, 0, 1, 1056, P, P), (P, 32, 0, 1, 0, P, P)])
def test_rows8_refuses(blank, rows, stride, dt, n, dim, codes, exps):
    lib, ctx = fs.load_library(), ctypes.addressof(blank)
    refused(lib.fs_rows_pack8(ctx, rows, stride, dt, n, dim, codes, exps, None))
    assert "pack8" in error(blank)
    refused(lib.fs_rows_unpack8(ctx, codes, exps, n, dim, rows, stride, dt, None))
    assert "unpack8" in error(blank)


def heads(**changes):
    rec = fs.fs_attention_args(q_stride=128, k_stride=64, v_stride=64, n_q=10, n_kv=20, batch=3, heads=4, kv_heads=2, head_dim=32,
                               dt=fs.FS_BF16, causal=1, max_q=0, scale=0.2, num_buckets=8, num_distances=30, dq_stride=128, dk_stride=64,
                               dv_stride=64, work_bytes=1 << 30)
    for name in ("q", "k", "v", "q_offsets", "kv_offsets", "kv_lengths", "bias", "bucket_of", "out", "out_f32", "lse", "dout", "dq",
                 "dk", "dv", "dbias", "work"):
        setattr(rec, name, P)
    for k, v in changes.items():
        setattr(rec, k, v)
    return rec


ATTENTION = [dict(n_q=-1), dict(n_kv=-1), dict(batch=-1), dict(batch=0), dict(max_q=-1), dict(heads=0), dict(kv_heads=0), dict(heads=3),
             dict(heads=-4, kv_heads=-2), dict(heads=2048, kv_heads=1024, q_stride=1 << 20, k_stride=1 << 20, v_stride=1 << 20),
             dict(head_dim=0), dict(head_dim=36, q_stride=160), dict(head_dim=136, q_stride=1 << 12, k_stride=1 << 12, v_stride=1 << 12),
             dict(dt=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=0.0), dict(scale=-0.2), dict(q_stride=(1 << 22) + 8), dict(k_stride=1 << 40), dict(causal=2), dict(bucket_of=None), dict(num_buckets=0),
             dict(num_buckets=1025), dict(num_distances=0), dict(num_distances=4097), dict(n_kv=1 << 31), dict(batch=1 << 31),
             dict(n_q=1 << 62), dict(q_offsets=None), dict(kv_offsets=None), dict(q_stride=120), dict(k_stride=60), dict(v_stride=-64),
             dict(q_stride=132), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4),
             dict(out=P + 8), dict(out_f32=P + 4)]


@pytest.mark.parametrize("changes", ATTENTION + [dict(max_q=1, work=None), dict(max_q=1, work_bytes=8), dict(max_q=1, work=P + 4)])
def test_jagged_attention_refuses(blank, changes):
    refused(fs.load_library().fs_jagged_attention(ctypes.addressof(blank), ctypes.byref(heads(**changes)), None))
    assert "jagged attention" in error(blank)


@pytest.mark.parametrize("changes", ATTENTION + [dict(dout=None), dict(dq=None), dict(lse=None), dict(dk=None), dict(dv=None),
                                                 dict(dq_stride=120), dict(dk_stride=66), dict(dv_stride=0), dict(dout=P + 8),
                                                 dict(dq=P + 8), dict(dk=P + 8), dict(dv=P + 8), dict(work=None), dict(work_bytes=8),
                                                 dict(work=P + 8)])
def test_jagged_attention_backward_refuses(blank, changes):
    refused(fs.load_library().fs_jagged_attention_backward(ctypes.addressof(blank), ctypes.byref(heads(**changes)), None))
    assert "jagged attention" in error(blank)


def test_attention_without_records_and_rows(blank):
    lib, ctx = fs.load_library(), ctypes.addressof(blank)
    for call in (lib.fs_jagged_attention, lib.fs_jagged_attention_backward):
        refused(call(None, ctypes.byref(heads()), None))
        refused(call(ctx, None, None))
    assert lib.fs_jagged_attention(ctx, ctypes.byref(heads(n_q=0)), None) == fs.FS_OK
    assert lib.fs_jagged_attention(ctx, ctypes.byref(heads(n_q=0, n_kv=0, batch=0)), None) == fs.FS_OK
    for size in (lib.fs_jagged_attention_work_bytes, lib.fs_jagged_attention_backward_work_bytes):
        assert size(None) == 0 and size(ctypes.byref(heads(heads=3))) == 0
    assert lib.fs_jagged_attention_work_bytes(ctypes.byref(heads())) == 0
    assert lib.fs_jagged_attention_work_bytes(ctypes.byref(heads(max_q=9))) == 0       # 18 columns: the other form
    few = lib.fs_jagged_attention_work_bytes(ctypes.byref(heads(max_q=2)))
    assert few > 0 and lib.fs_jagged_attention_work_bytes(ctypes.byref(heads(max_q=2, n_kv=20_000))) > few
    assert lib.fs_jagged_attention_backward_work_bytes(ctypes.byref(heads(dbias=None))) < \
        lib.fs_jagged_attention_backward_work_bytes(ctypes.byref(heads()))


class Stub:
    """A context for the checks of the binding, which come before the library is called."""
    device, handle = 0, None
    lib = None

    def check(self, rc, where):
        raise AssertionError("reached the library")


@pytest.mark.parametrize("changes", [
    dict(),                                                                                   # not on the GPU
    dict(k=torch.zeros(7, 2, 8)), dict(v=torch.zeros(7, 2, 16).transpose(0, 1)), dict(q=torch.zeros(7, 16)),
    dict(q=torch.zeros(7, 2, 16).half()), dict(k=torch.zeros(7, 2, 16).bfloat16()), dict(q=torch.zeros(7, 2, 32)[:, :, ::2]),
    dict(q=torch.zeros(7, 4, 16)[:, ::2]), dict(q_offsets=torch.zeros(4, dtype=torch.int32)),
    dict(kv_offsets=torch.zeros(5, dtype=torch.int64)), dict(kv_lengths=torch.zeros(4, dtype=torch.int64)),
    dict(bias=torch.zeros(4, 3)), dict(bias=torch.zeros(4, 2).double()), dict(bucket_of=torch.zeros(4, dtype=torch.int64)),
    dict(causal=False, bucket_of=torch.zeros(4, dtype=torch.int32)), dict(out={"out": torch.zeros(7, 2, 8)}),
    dict(out={"lse": torch.zeros(7, 2)})])
def test_binding_refuses_attention(changes):
    args = dict(q=torch.zeros(7, 2, 16), k=torch.zeros(7, 2, 16), v=torch.zeros(7, 2, 16), q_offsets=torch.zeros(4, dtype=torch.int64),
                kv_offsets=torch.zeros(4, dtype=torch.int64), bias=torch.zeros(4, 2), bucket_of=torch.zeros(4, dtype=torch.int32))
    with pytest.raises((ValueError, TypeError)):
        fs.fs_jagged_attention(Stub(), **{**args, **changes})


@pytest.mark.parametrize("call", [
    lambda c, x, w: fs.fs_block_norm(c, x, w_pre=w),                                          # not on the GPU
    lambda c, x, w: fs.fs_block_norm(c, x.t(), w_pre=torch.ones(3)),                          # columns apart
    lambda c, x, w: fs.fs_block_norm(c, x, x, x[:2], w, w, w),                                # another number of rows
    lambda c, x, w: fs.fs_block_norm(c, x, x, x.double(), w, w, w),                           # another type
    lambda c, x, w: fs.fs_block_norm(c, x.half(), w_pre=w),
    lambda c, x, w: fs.fs_block_norm(c, x, w_pre=w[:5]),
    lambda c, x, w: fs.fs_block_norm(c, x, w_pre=w, pack=("a",)),
    lambda c, x, w: fs.fs_block_norm(c, x, w_pre=w, pack=("q",)),
    lambda c, x, w: fs.fs_block_norm_backward(c, x, x, y=x[:2], w_pre=w),
    lambda c, x, w: fs.fs_block_norm_backward(c, x, x, y=fs.Rows8(x, x), w_pre=w),
    lambda c, x, w: fs.fs_rows_pack8(c, x.t()),
    lambda c, x, w: fs.fs_rows_unpack8(c, fs.Rows8(x.to(torch.int8), torch.zeros(3, 2, dtype=torch.uint8))),
])
def test_binding_refuses(call):
    with pytest.raises((ValueError, TypeError)):
        call(Stub(), torch.zeros(3, 32), torch.ones(32))
