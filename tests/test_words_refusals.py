"""The words entry points refuse wrong calls before any launch (no GPU needed: sizes, types,
alignment and the rules' completeness are checked before the device is asked, and without a
GPU no pointer is device memory).  The state is a zeroed block that no refused call reads."""
import ctypes as C

import pytest

from paper_1510_06549_amd import spdp as sp

BLOCK = C.create_string_buffer(1 << 16)
STATE = C.c_void_p((C.addressof(BLOCK) + 255) // 256 * 256)
P = 1 << 20  # an aligned address that is never read


def rows8(rows=4, cols=200, q=P, e=P):
    return sp._Rows8(rows, cols, q, e)


def refused(rc, text):
    msg = sp.spdp_last_error()
    assert rc == sp.SPDP_E_ARG and text in msg, (rc, msg)


def rules(**kw):
    r = sp._Rules(rows=4, n_words=100, n_bias=1, n_masks=1, n_listed=9)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("kw,text", [
    (dict(out=None), "out is NULL"),
    (dict(type=sp.SPDP_F16), "SPDP_F64 or SPDP_F32"),
    (dict(type=7), "SPDP_F64 or SPDP_F32"),
    (dict(out=rows8(rows=-1)), "0 <= rows < 2^31"),
    (dict(out=rows8(cols=0)), "1 <= cols < 2^24"),
    (dict(out=rows8(cols=1 << 24)), "1 <= cols < 2^24"),
    (dict(out=rows8(q=P + 8)), "not 16-byte aligned"),
    (dict(out=rows8(q=None)), "out is NULL"),
    (dict(out=rows8()), "out is not device memory"),
    (dict(ld=199, out=rows8(rows=0)), "overlap at ld = 199"),
])
def test_pack8(kw, text):
    a = dict(x=P, type=sp.SPDP_F64, ld=200, out=rows8())
    a.update(kw)
    out = a["out"] and C.addressof(a["out"])
    refused(sp.lib().spdp_pack8(STATE, a["x"], a["type"], a["ld"], out), text)


@pytest.mark.parametrize("kw,text", [
    (dict(a=None), "a is NULL"),
    (dict(b=None), "b is NULL"),
    (dict(a=rows8(rows=0, cols=100)), "100 and 200 columns"),
    (dict(type=sp.SPDP_F64), "SPDP_F32, SPDP_F16 or SPDP_BF16"),
    (dict(a=rows8(rows=1 << 31)), "0 <= rows < 2^31"),
])
def test_product8(kw, text):
    a = dict(a=rows8(rows=0), b=rows8(rows=0), type=sp.SPDP_F32, ld=100)
    if "type" in kw:
        a["b"] = None
    a.update(kw)
    if a["type"] == sp.SPDP_F64:
        # (the type is looked at where there is something to write: rules of the scores)
        refused(sp.lib().spdp_top(STATE, P, 100, a["type"], 4, 100, None, 1, P, P, P, 0), text)
        return
    ref = lambda r: r and C.addressof(r)  # noqa: E731
    refused(sp.lib().spdp_product8(STATE, ref(a["a"]), ref(a["b"]), 0, P, a["type"], a["ld"]),
            text)


@pytest.mark.parametrize("kw,text", [
    (dict(rules=None), "rules is NULL"),
    (dict(ldx=99), "x: rows of 100 elements overlap"),
    (dict(type=sp.SPDP_F64), "SPDP_F32, SPDP_F16 or SPDP_BF16"),
    (dict(rules=rules(rows=-1)), "0 <= rows"),
    (dict(rules=rules(rows=1 << 31)), "0 <= rows"),
    (dict(rules=rules(n_words=0)), "1 <= n_words"),
    (dict(ldx=1 << 62), "more elements than memory holds"),
    (dict(x=P + 1), "x is misaligned"),
    (dict(), "x is not device memory"),
    (dict(x=None), "x is NULL"),
    (dict(rules=rules(rows=0, n_listed=-1)), "negative size"),
    (dict(rules=rules(rows=0, n_bias=-1)), "negative size"),
])
def test_adjust(kw, text):
    a = dict(x=P, ldx=100, y=P, ldy=100, type=sp.SPDP_F32, rules=rules())
    a.update(kw)
    ref = a["rules"] and C.addressof(a["rules"])
    refused(sp.lib().spdp_adjust(STATE, a["x"], a["ldx"], a["y"], a["ldy"], a["type"], ref), text)


@pytest.mark.parametrize("kw,text", [
    (dict(rules=rules(rows=3)), "rules for 3 x 100 scores"),
    (dict(rules=rules(n_words=99)), "rules for 0 x 99 scores"),
    (dict(k=0), "k must be in [1, 256]"),
    (dict(k=257), "k must be in [1, 256]"),
    (dict(rows=-1), "0 <= rows"),
    (dict(n=0), "1 <= n_words"),
    (dict(work=P + 8), "not 16-byte aligned"),
    (dict(work_bytes=-1), "a workspace of"),
])
def test_top(kw, text):
    a = dict(rows=0, n=100, rules=None, k=3, work=P, work_bytes=0)
    a.update(kw)
    if a["rules"] is not None and a["rules"].rows == 4:
        a["rules"].rows = 0
    ref = a["rules"] and C.addressof(a["rules"])
    refused(sp.lib().spdp_top(STATE, P, max(a["n"], 100), sp.SPDP_F32, a["rows"], a["n"], ref,
                              a["k"], P, P, a["work"], a["work_bytes"]), text)


@pytest.mark.parametrize("kw,text", [
    (dict(draws=-1), "draws must be in"),
    (dict(draws=(1 << 20) + 1), "draws must be in"),
    (dict(temperature=0.0), "temperature must be in"),
    (dict(temperature=float("nan")), "temperature must be in"),
    (dict(temperature=1e7), "temperature must be in"),
    (dict(work=P + 8), "not 16-byte aligned"),
])
def test_draw(kw, text):
    a = dict(draws=3, temperature=1.0, work=P)
    a.update(kw)
    refused(sp.lib().spdp_draw(STATE, P, 100, sp.SPDP_BF16, 0, 100, None, a["temperature"],
                               a["draws"], None, 0, 0, P, P, a["work"], 0), text)


def test_predict():
    L = sp.lib()
    a = sp._Answer(type=sp.SPDP_F32, temperature=1.0)
    docs, words = rows8(rows=0), rows8(rows=0)
    call = lambda d, w, x: L.spdp_predict(  # noqa: E731
        STATE, d and C.addressof(d), w and C.addressof(w), None, x and C.addressof(x), None, 0)
    refused(call(docs, words, None), "null argument")
    refused(call(None, words, a), "docs is NULL")
    refused(call(docs, None, a), "words is NULL")
    refused(call(docs, rows8(rows=0, cols=3), a), "200 and 3 columns")
    refused(call(docs, words, a), "no words")


def test_null_state_and_work_sizes():
    L = sp.lib()
    out = C.c_int64()
    for rc in (L.spdp_pack8(None, P, 0, 1, None), L.spdp_product8(None, None, None, 0, P, 1, 1),
               L.spdp_adjust(None, P, 1, P, 1, 1, None),
               L.spdp_top(None, P, 1, 1, 1, 1, None, 1, P, P, P, 0),
               L.spdp_draw(None, P, 1, 1, 1, 1, None, 1.0, 1, None, 0, 0, P, P, P, 0),
               L.spdp_predict(None, None, None, None, None, None, 0),
               L.spdp_words_work(1, 1, 1, None), L.spdp_words_work(-1, 1, 1, C.byref(out)),
               L.spdp_words_work(1, 0, 1, C.byref(out)), L.spdp_words_work(1, 1, -1, C.byref(out)),
               L.spdp_predict_work(1, 1, sp.SPDP_F64, 1, C.byref(out)),
               L.spdp_predict_work(1, 1, sp.SPDP_F32, 257, C.byref(out))):
        assert rc == sp.SPDP_E_ARG
    # more rows, words or places need no less room
    size = lambda *a: sp.spdp_words_work(*a)  # noqa: E731
    assert size(0, 100, 10) == 0
    for rows in (1, 7, 1000):
        for n in (1, 4096, 4097, 10 ** 6):
            assert size(rows, n, 256) >= size(rows, n, 10) >= size(rows, n, 0) > 0
            assert size(rows + 1, n, 10) >= size(rows, n, 10)


def test_binding_wants_device_tensors():
    import torch

    x = torch.zeros(4, 200)
    with pytest.raises(ValueError):
        sp.spdp_adjust(STATE, x, None, x)
    with pytest.raises(ValueError):
        sp.Rows8(torch.zeros(4, 256, dtype=torch.float8_e4m3fn),
                 torch.zeros(4, 2, dtype=torch.uint8), 200)
    with pytest.raises(ValueError):
        sp.Rules(4, 100, bias=torch.zeros(1, 100))


@pytest.mark.parametrize("type,ld,text", [
    (sp.SPDP_F64, 100, "SPDP_F32, SPDP_F16 or SPDP_BF16"),
    (7, 100, "SPDP_F32, SPDP_F16 or SPDP_BF16"),
    (-1, 0, "SPDP_F32, SPDP_F16 or SPDP_BF16"),
    (sp.SPDP_F32, -1, "c: rows of 0 elements overlap at ld = -1"),
])
def test_product8_without_words(type, ld, text):
    """A wrong call is refused where there is nothing to write, too."""
    none = rows8(rows=0)
    call = lambda *a: sp.lib().spdp_product8(  # noqa: E731
        STATE, C.addressof(none), C.addressof(none), 0, P, *a)
    refused(call(type, ld), text)
    assert call(sp.SPDP_F16, 0) == sp.SPDP_OK


def test_binding_predict_wants_counts():
    import numpy as np

    s = object.__new__(sp.Sampler)
    s.h = None
    for kw in (dict(top=-1), dict(draws=-1), dict(top=5, draws=-2)):
        for rows in (0, 2):
            with pytest.raises(ValueError, match="how many words"):
                s.predict(np.ones((rows, 3)), np.ones((5, 3)), **kw)


class TwoDevices:
    """What Sampler.predict asks of the library, with the device that is current recorded: the
    state's is 1."""

    def __init__(self, error=0):
        self.device, self.error, self.mine, self.elsewhere, self.at = 0, error, 0, [], 1 << 20

    def __getattr__(self, name):
        def call(*args):
            if self.device == 1:
                self.mine += 1
            else:
                self.elsewhere.append(name)
            if name == "hipMalloc":
                self.at += 1 << 20
                args[0]._obj.value = self.at
            elif name == "spdp_predict_work":
                args[-1]._obj.value = 64
            elif name == "spdp_predict":
                return self.error
            elif name == "spdp_last_error":
                return b"refused"
            return 0

        return call

    def hipGetDevice(self, out):
        out._obj.value = self.device
        return 0

    def hipSetDevice(self, device):
        self.device = device.value
        return 0


@pytest.mark.parametrize("error", [0, sp.SPDP_E_ARG])
def test_binding_predict_on_the_states_device(monkeypatch, error):
    """Memory comes from the device that the state was made on, whichever is current."""
    import numpy as np

    lib = TwoDevices(error)
    monkeypatch.setattr(sp, "lib", lambda: lib)
    s = object.__new__(sp.Sampler)
    s.h, s.device = None, 1
    call = lambda: s.predict(np.ones((2, 3)), np.ones((5, 3)), top=2, draws=1)  # noqa: E731
    if error:
        with pytest.raises(sp.SpdpError, match="refused"):
            call()
    else:
        assert [x.shape for x in call()] == [(2, 2), (2, 2), (2, 1), (2, 1)]
    assert lib.device == 0 and lib.mine > 10
    assert set(lib.elsewhere) <= {"hipFree"}


@pytest.mark.parametrize("kw", [dict(allowed=True), dict(allowed=[True]), dict(allowed=[True] * 4),
                                dict(allowed=[[True] * 5] * 2), dict(bias=[0.5])])
def test_binding_predict_wants_whole_tables(monkeypatch, kw):
    """One truth value is not one for every word."""
    import numpy as np

    lib = TwoDevices()
    monkeypatch.setattr(sp, "lib", lambda: lib)
    s = object.__new__(sp.Sampler)
    s.h, s.device = None, 1
    with pytest.raises(ValueError, match="reshape"):
        s.predict(np.ones((2, 3)), np.ones((5, 3)), top=2, **kw)
    s.predict(np.ones((2, 3)), np.ones((5, 3)), top=2, allowed=[1, 0, 1, 0, 1], bias=range(5))
