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


@pytest.mark.parametrize("record", ["fs_block_args"])
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


class Stub:
    """A context for the checks of the binding, which come before the library is called."""
    device, handle = 0, None
    lib = None

    def check(self, rc, where):
        raise AssertionError("reached the library")


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
