"""What the dense product's entry points take and launch (tests/dense_recorder.cpp), on the host: every shape within the documented limits, in a
launch of fewer than 2^32 lanes whose tiles cover it; what is beyond them is refused."""
import ctypes
import os
import subprocess

import pytest

from paper_2401_14110_amd import binding as lb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUF, LARGE = 1 << 20, 1 << 46        # (never read: an address on a 256-byte boundary), a workspace's size
ROWS, THREADS = (256, 128, 64, 192, 128, 64, 256, 128, 64), (512, 256, 256, 512, 256, 256, 512, 256, 256)
COLS = (256, 128, 64, 256, 128, 64, 256, 128, 64)


class Record(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int32), ("products", ctypes.c_int32), ("tiles", ctypes.c_int64), ("beside", ctypes.c_int64)]


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("launches") / "dense_recorder.so")
    csrc = os.path.join(ROOT, "paper_2401_14110_amd", "csrc")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared",
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
                    "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "lba_dense.hip"), os.path.join(csrc, "lba_norm.hip"),
                    "-x", "hip", os.path.join(ROOT, "tests", "dense_recorder.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    vp, i64, i32, fmt, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, lb.lba_infmt, ctypes.c_size_t
    lib.lba_dense.argtypes = [vp, vp, i64, i64, i64, fmt, fmt, i32, vp, i32, lb.lba_drop, vp, i32, vp, i32, fmt, vp, size, vp]
    lib.lba_dense_bwd.argtypes = [vp, i32, vp, vp, i64, i64, i64, fmt, fmt, i32, vp, i32, lb.lba_drop, vp, vp, vp, vp, size, vp]
    return lib


def launches(lib, rc):
    out = (Record * 2)()
    n = lib.take_launches(out)
    assert (rc == lb.ERR_SHAPE) == (n == 0), (rc, n)           # (without a device the last error need not be none)
    return None if rc == lb.ERR_SHAPE else list(out[:n])


def forward(lib, M, N, K, fmt=(4, 3, 7), gated=0):
    f, d = lb.lba_infmt(*fmt), lb.lba_drop(0.0, 0, 0, None)
    return launches(lib, lib.lba_dense(BUF, BUF, M, N, K, f, f, gated, None, 0, d, None, 0, BUF, 2, f, BUF, LARGE, None))


def backward(lib, M, N, K, g_type=1, gated=0):
    f, d = lb.lba_infmt(4, 3, 7), lb.lba_drop(0.0, 0, 0, None)
    return launches(lib, lib.lba_dense_bwd(BUF, g_type, BUF, BUF, M, N, K, f, f, gated, None, 0, d, BUF, BUF, None, BUF, LARGE, None))


def up(x, m):
    return (x + m - 1) // m


def covers(r, M, cols, slices=1):
    return r.tiles >= up(M, ROWS[r.tile]) * up(cols, COLS[r.tile]) and (r.tiles + r.beside) * THREADS[r.tile] < 1 << 32


@pytest.mark.parametrize("fmt", [(4, 3, 7), (3, 4, 5)])
@pytest.mark.parametrize("M,N,K,gated", [
    (1 << 27, 32, 32, 0), (1 << 30, 1, 16, 0), (1 << 17, 1 << 20, 32, 0), (1 << 30, 256, 16, 0), (1 << 13, 1 << 20, 32, 0), (1 << 30, 128, 64, 1),
    ((1 << 23) - 255, 65000, 16, 0), (65, 1 << 20, 1 << 30, 0), (1 << 18, 1 << 20, 16, 1), (1 << 19, 1 << 20, 16, 0), (3985, 770, 768, 0)])
def test_forward_within_the_limits(rec, M, N, K, gated, fmt):
    cols = 2 * N if gated else N
    got = forward(rec, M, N, K, fmt, gated)
    if up(M, 256) * up(cols, 256) < 1 << 23:
        assert len(got) == 1 and covers(got[0], M, cols)
    else:
        assert got is None


@pytest.mark.parametrize("gated", [0, 1])
def test_forward_at_the_limit(rec, gated):
    N = (1 << 20) >> gated
    assert forward(rec, (1 << 19) - 256, N, 16, gated=gated) is not None and forward(rec, (1 << 19) - 255, N, 16, gated=gated) is None
    assert forward(rec, 1 << 30, 256 >> gated, 16, gated=gated) is not None and forward(rec, 1 << 30, 257, 16, gated=gated) is None
    assert len(forward(rec, 64, N, 1 << 30, gated=gated)) == 1                  # few rows: their own kernel


@pytest.mark.parametrize("g_type", [0, 1])
@pytest.mark.parametrize("M,N,K,gated", [
    (1 << 25, 32, 32, 0), (64000000, 1, 3, 0), (1 << 18, 1 << 14, 32, 0), (1 << 18, 1 << 13, 32, 1), (1, 1 << 20, 4000, 0), (7, 1 << 20, 1900, 1),
    ((1 << 26) - 1000, 100, 0, 0), (1 << 30, 128, 0, 0), (64, 8, 60000000 // 2, 0), (3985, 770, 771, 0)])
def test_backward_within_the_limits(rec, M, N, K, gated, g_type):
    cols = 2 * N if gated else N
    assert (M + 64) * (K + 64) <= 1 << 32 or K == 0
    got = backward(rec, M, N, K, g_type, gated)
    if (M + 64) * (K + 64) > 1 << 32 or (cols + 64) * (K + 64) > 1 << 32 or up(M, 128) * up(cols, 128) >= 3 << 22:
        assert got is None
        return
    assert covers(got[0], M, cols) and len(got) == (2 if K else 1)
    if K:
        r = got[1]
        assert r.products == 2 and (r.tiles + r.beside) * THREADS[r.tile] < 1 << 32
        assert r.tiles >= up(M, ROWS[r.tile]) * up(K, COLS[r.tile]) + up(cols, ROWS[r.tile]) * up(K, COLS[r.tile])


def test_backward_at_the_limit(rec):
    # rows of B and of A times few codes of k: tiles of 128 x 128 outputs, fewer than 3 * 2^22
    M = 3 << 16
    assert up(M, 128) * up(1 << 20, 128) == 3 << 22 and (M + 64) * (16 + 64) < 1 << 32
    assert backward(rec, M, 1 << 20, 16) is None and backward(rec, M - 128, 1 << 20, 16) is not None
