"""Sizes that the words entry points check behind the device's answers (no GPU needed): a
child process loads stand-ins for the calls that ask for an allocation's extent before the
library, so that every address is inside one of 2^62 bytes.  The current device is not to be
had there, so that no call that is not refused can launch anything."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = """
#include <stddef.h>
int hipMemGetAddressRange(void **base, size_t *size, void *p)
{
    (void)p;
    *base = 0;
    *size = (size_t)1 << 62;
    return 0;
}
int hipGetDeviceCount(int *n) { *n = 1; return 0; }
int hipGetDevice(int *device) { (void)device; return 100; }
"""

HEAD = """
import ctypes as C, sys
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
from paper_1510_06549_amd import spdp as sp
L, P = sp.lib(), 1 << 20
BLOCK = C.create_string_buffer(1 << 16)
STATE = C.c_void_p((C.addressof(BLOCK) + 255) // 256 * 256)
def refused(rc, text):
    assert rc == sp.SPDP_E_ARG and text in sp.spdp_last_error(), (rc, sp.spdp_last_error())
def accepted(rc):  # (up to the device that is not there)
    assert rc == sp.SPDP_E_HIP, (rc, sp.spdp_last_error())
"""


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    at = tmp_path_factory.mktemp("stand_in")
    (at / "s.c").write_text(STAND_IN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(at / "s.so"), str(at / "s.c")], check=True)
    return str(at / "s.so")


def run(stand_in, code):
    done = subprocess.run([sys.executable, "-c", HEAD + code, stand_in], cwd=ROOT,
                          capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-2000:]


def test_predict_of_more_scores_than_64_bits_count(stand_in):
    """Documents and words of one buffer can be 2^31 each: a workspace for some of their scores
    is one for fewer documents at a time, and one too small for a document is refused."""
    run(stand_in, """
for n in ((1 << 31) - 1, 3 << 29, 1 << 20, 1000):
    rows = sp._Rows8(n, 5, P, P)
    for type in (sp.SPDP_F32, sp.SPDP_F16, sp.SPDP_BF16):
        a = sp._Answer(type=type, k=1, top_word=P, top_value=P, temperature=1.0)
        one = -(-n * (4 if type == sp.SPDP_F32 else 2) // 256) * 256 + sp.spdp_words_work(1, n, 1)
        call = lambda have: L.spdp_predict(STATE, C.addressof(rows), C.addressof(rows), None,
                                           C.addressof(a), P, have)
        for have in (0, 1 << 10, one - 256):
            refused(call(have), f"a workspace of {one} bytes, not {have}")
        accepted(call(one))
        accepted(call(1 << 40))
""")


def test_workspaces_of_their_own(stand_in):
    """Best words do not ask for the room that only draws use, nor draws for keys."""
    run(stand_in, """
for rows, n, k in ((20000, 100000, 10), (1, 100000, 1), (1024, 5000, 256), (1000000, 3, 256)):
    ld, f32 = n, sp.SPDP_F32
    top = lambda have: L.spdp_top(STATE, P, ld, f32, rows, n, None, k, P, P, P, have)
    draw = lambda have: L.spdp_draw(STATE, P, ld, f32, rows, n, None, 1.0, 7, None, 0, 0, P, P, P, have)
    both = sp.spdp_words_work(rows, n, k)
    own = (min(both, 8 * k * (rows + 1024) + 256), min(both, 5136 * rows * -(-n // 8192) + 512))
    for call, have in zip((top, draw), own):
        accepted(call(both))
        accepted(call(have))
        refused(call(0), "a workspace of")
    assert both <= max(8 * k * (rows + 1024) + 256, 5136 * rows * -(-n // 8192) + 512)
""")
