"""CPU checks of the linear layers' entry points at the ends of what their documentation allows."""
import os
import subprocess
import sys

import pytest

from paper_2208_00763_b200 import binding as hk
from paper_2208_00763_b200 import build as lib_build

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
