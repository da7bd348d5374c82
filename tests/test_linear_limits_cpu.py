"""CPU checks of the linear layers' entry points at the ends of what their documentation allows."""
import os
import re
import subprocess
import sys

import pytest

from paper_2208_00763_b200 import binding as hk
from paper_2208_00763_b200 import build as lib_build
from test_linear_cpu import BIAS, C, F, OFF, OUT, RES, SCALE, SCALE2, W, X, call, space

TESTS = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module", autouse=True)
def built_library():
    lib_build.build()
    return hk.lib()


def without_devices(code):
    """What `code` prints in a process that sees no device: calls that nothing refuses go on up to their launch, which fails."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="", PYTHONPATH=os.pathsep.join([TESTS, os.path.dirname(TESTS)]))
    done = subprocess.run([sys.executable, "-c", "from test_linear_cpu import *\n" + code], env=env, capture_output=True, text=True)
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])
    return done.stdout.split()


def test_depths_next_to_the_largest():
    # unsigned 1-bit codes, one per byte, and dense where the depth fills whole bytes
    depths = [2 ** 31 - less for less in (129, 128, 127, 112, 16, 8, 1)]
    made = without_devices("""
for K in %s:
    for store in (8, 1)[:2 - (K %% 8 > 0)]:
        a = dict(M=17, N=128, K=K, p=1, q=1, xs=0, ws=0, store=store, x_row=1 << 31, x=1 << 50, out_row=128, out=1 << 40, w=1 << 52, ep=S,
                 ws_ptr=1 << 54, ws_bytes=1 << 53)
        print(call(**a), call(grouped=True, E=1, offsets=1 << 41, **a), call(**{**a, 'M': 1, 'N': 1}), flush=True)
""" % depths)
    assert made == [str(hk.ERR_CUDA)] * 3 * (len(depths) + sum(K % 8 == 0 for K in depths))


def test_the_workspace_overlaps_no_operand():
    # a layer whose rows are copied; every operand that the kernels still read or write after the copy, its first and its last byte
    M, N, K, E = 100, 32, 60, 3
    ep = dict(F, d_x_scale=SCALE, d_w_scale=SCALE2, d_bias=BIAS, d_residual=RES, residual_row_stride=40)
    for grouped in (False, True):
        columns = N * (E if grouped else 1)
        big = dict(M=M, N=N, K=K, x_row=60, ep=ep)
        need = M * 64 + columns * 64
        assert space(**big, E=E if grouped else 0) == need
        ends = [(SCALE, M * 4), (SCALE2, columns * 4), (BIAS, columns * 4), (RES, (M - 1) * 80 + N * 2), (X, (M - 1) * 60 + K), (W, columns * K),
                (OUT, (M - 1) * 64 + N * 2)] + ([(OFF, (E + 1) * 4)] if grouped else [])
        for at, size in ends:
            first_behind = -(-(at + size) // 16) * 16
            for ptr in (at - need + 16, at, first_behind - 16):
                assert call(grouped=grouped, E=E, **big, ws_ptr=ptr, ws_bytes=need) == hk.ERR_INVALID_ARG, (grouped, hex(at), hex(ptr))


def test_a_workspace_behind_or_beside_what_is_used_is_fine():
    M, N, K = 100, 32, 60
    ep = dict(F, d_x_scale=SCALE, d_bias=BIAS)
    need = M * 64 + N * 64
    # next to an operand; with an operand behind the bytes that the call needs; and none of it needed
    made = without_devices("""
ep = dict(F, d_x_scale=SCALE, d_bias=BIAS)
big = dict(M=%d, N=%d, K=%d, x_row=60, ep=ep)
print(call(**big, ws_ptr=SCALE - %d, ws_bytes=%d), call(**big, ws_ptr=SCALE - %d, ws_bytes=1 << 30), call(ep=ep, ws_ptr=SCALE, ws_bytes=1 << 20))
""" % (M, N, K, need, need, need))
    assert made == [str(hk.ERR_CUDA)] * 3


def test_columns_of_one_buffer():
    # bf16 rows of 64 bytes, 128 apart, four of them: the residual's lie between the output's, or in front or behind, or share a value
    apart = [64, -64, 64 - 3 * 128, 64 + 2 * 128, 66 + 3 * 128, -66 - 3 * 128]
    shared = [62, 66, -62, -66, 128, 66 - 3 * 128, 62 + 3 * 128]
    for off in shared:
        for grouped in (False, True):
            assert call(grouped=grouped, out_row=64, ep=dict(F, d_residual=OUT + off, residual_row_stride=64)) == hk.ERR_INVALID_ARG, off
    made = without_devices("for off in %s:\n"
                           "    print(*(call(grouped=g, out_row=64, ep=dict(F, d_residual=OUT + off, residual_row_stride=64)) for g in (False, True)))" % apart)
    assert made == [str(hk.ERR_CUDA)] * 2 * len(apart)


def test_columns_of_one_buffer_with_other_strides():
    # rows 128 and 130 bytes apart meet somewhere, or may
    for off in (0, 64, -64):
        assert call(out_row=64, ep=dict(F, d_residual=OUT + off, residual_row_stride=65)) == hk.ERR_INVALID_ARG
    # codes next to the codes they come from: 64 bytes of x, 32 of out, 96 apart
    for off in (63, -31, 65, 96, 0):
        assert call(x_row=96, out=X + off, out_row=96, ep=dict(C, hi=1)) == hk.ERR_INVALID_ARG
    made = without_devices("print(*(call(x_row=96, out=X + off, out_row=96, ep=dict(C, hi=1)) for off in (64, -32, 64 + 96)))")
    assert made == [str(hk.ERR_CUDA)] * 3


def test_what_the_linear_kernels_read_they_read_with_ordinary_loads():
    # they are launched while the kernel before may still write; the read-only path promises data that stays constant meanwhile
    csrc = os.path.join(os.path.dirname(TESTS), "paper_2208_00763_b200", "csrc")
    for name in ("hikonv_linear_util.cuh", "hikonv_linear_rows.cu", "hikonv_linear_tc.cu", "hikonv_quantize.cu"):
        text = re.sub(r"//.*", "", open(os.path.join(csrc, name)).read())
        assert not re.search(r"__ldg\(|ld\.global\.nc|__ldc[sagv]\(|const\s+\w+\s*\*\s*__restrict__", text), name
