"""Words of documents on the GPU against the fp64 oracle (oracle/words.py): 8-bit rows and
their products, rules on scores, best words, draws, and all of them in one call.

Tolerances.  Packed rows, adjusted scores, best words and drawn words are equal to the
oracle's: a packed value and a rule's step are one rounding each of exact inputs, and a draw
is compared unless its uniform lies within 1e-11 of a border between two words (the borders
are sums of up to 10^5 fp64 weights, each off by a few 2^-53 of the total at most).  A
product's sum of P padded columns takes at most P roundings of 2^-23 of the sum of
magnitudes (2^-24, or a cut of the last place); its logarithm adds 2^-22 of itself (the
hardware's base-2 logarithm, its scaling and their roundings); then half a step of the
output's type.
"""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle
import synth
from oracle import words as ow
from paper_1510_06549_amd import spdp as sp

pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def say(*a):
    print(*a, flush=True)


def _state(stream=None):
    return sp.Sampler(np.array([0, 1], np.int32), np.array([0, 2], np.int64),
                      np.array([0], np.int32), 1, 2, 1, 0.1, 0.5, 1.0, 0.1,
                      hip_stream=None if stream is None else stream.cuda_stream)


@pytest.fixture(scope="module")
def state():
    s = _state()
    yield s
    s.close()


def dev(x, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(x)).to("cuda", dtype)


def framed(rows, cols, dtype, ld=None, at=0, fill=7.0):
    """(a [rows, cols] view at element `at` of a buffer with rows `ld` apart, the buffer)."""
    ld = cols if ld is None else ld
    buf = torch.full((at + rows * ld + 64,), fill, dtype=dtype, device="cuda")
    return buf[at:at + rows * ld].view(rows, ld)[:, :cols], buf


def frame_kept(buf, view, fill=7.0):
    """Whether everything of the buffer outside the view is as it was."""
    other = buf.clone()
    torch.as_strided(other, view.shape, view.stride(), view.storage_offset()).fill_(fill)
    return bool((other.float() == fill).all())


def work_for(rows, n, take=0):
    return torch.empty(max(16, sp.spdp_words_work(rows, n, take)), dtype=torch.uint8,
                       device="cuda")


# ---------------------------------------------------------------------------
# rows in 8 bits
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("type", ["f64", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 50, 0), (2, 128, 1), (5, 129, 0),
                                           (9, 500, 3), (2, 1000, 0), (70, 257, 0)])
def test_pack(state, rows, cols, pad, type):
    say(f"pack {rows} x {cols} + {pad} {type}")
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=(rows, cols)) * 6)
    x[rng.random(x.shape) < 0.1] = 0
    x[:, 0] = 448.0 if rows > 2 else 3.0
    if rows >= 3:
        # ties between neighbouring codes, values of every kind that has no number
        mid = (ow.VALUES8[:-1] + ow.VALUES8[1:]) / 2
        n = min(cols - 1, 126)
        x[1, 1:1 + n] = mid[-n:] if cols < 60 else mid[:n]
        x[2, :cols // 2] = [np.nan, np.inf, -np.inf, 1e-30, -2.0][:cols // 2] + \
            [0.5] * max(0, cols // 2 - 5)
    if rows >= 5:
        x[3] = 0.0
        x[4] *= 1e-35
    x = dev(x, TYPES[type])
    src, _ = framed(rows, cols, TYPES[type], ld=cols + pad, at=pad)
    src.copy_(x)
    nb = -(-cols // 128)
    qbuf = torch.full((rows * nb * 128 + 256,), 0x55, dtype=torch.uint8, device="cuda")
    ebuf = torch.full((rows * nb + 64,), 0x55, dtype=torch.uint8, device="cuda")
    out = sp.Rows8(qbuf[:rows * nb * 128].view(rows, -1).view(torch.float8_e4m3fn),
                   ebuf[:rows * nb].view(rows, nb), cols)
    sp.spdp_pack8(state.h, src, out)
    q, e = ow.pack8(src.double().cpu().numpy())
    np.testing.assert_array_equal(out.e.cpu().numpy(), e)
    got = out.q.view(torch.uint8).cpu().numpy()
    nan = (q & 127) == 127
    np.testing.assert_array_equal((got & 127) == 127, nan)
    # (a zero's sign is the value's, or +)
    np.testing.assert_array_equal(ow.value8(got)[~nan], ow.value8(q)[~nan])
    assert (qbuf[rows * nb * 128:] == 0x55).all() and (ebuf[rows * nb:] == 0x55).all()


def test_pack_rounds_once(state):
    """Values a hair above and below the middle of two codes: a rounding to fp32 first
    would make them ties."""
    say("pack, double rounding")
    mid = (ow.VALUES8[:-1] + ow.VALUES8[1:]) / 2
    x = np.concatenate([[448.0], mid[:126], [0.0], [448.0], mid[:126] * (1 + 2.0 ** -40), [0.0],
                        [448.0], mid[:126] * (1 - 2.0 ** -40)])[None]
    out = sp.Rows8.empty(1, x.shape[1])
    sp.spdp_pack8(state.h, dev(x), out)
    q, e = ow.pack8(x)
    np.testing.assert_array_equal(out.q.view(torch.uint8).cpu().numpy(), q)


def test_pack_empty_and_extremes(state):
    say("pack, no rows; scales at both ends")
    sp.spdp_pack8(state.h, torch.empty((0, 9), dtype=torch.float64, device="cuda"),
                  sp.Rows8.empty(0, 9))
    x = np.array([[1e300, 1.0], [1e-300, 1e-310], [448 * 2.0 ** 127, -1.0], [2.0 ** -127, 0.0],
                  [-0.0, 5e-324]])
    out = sp.Rows8.empty(5, 2)
    sp.spdp_pack8(state.h, dev(x), out)
    q, e = ow.pack8(x)
    np.testing.assert_array_equal(out.e.cpu().numpy(), e)
    got = ow.value8(out.q.view(torch.uint8).cpu().numpy())
    np.testing.assert_array_equal(got, ow.value8(q))


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def _packed(rng, rows, cols, spread, sign=False):
    x = np.exp(rng.normal(size=(rows, cols)) * spread)
    if sign:
        x *= rng.choice([-1.0, 1.0], size=x.shape)
    x[rng.random(x.shape) < 0.05] = 0
    x *= np.exp(rng.normal(size=(rows, 1)) * 3)
    q, e = ow.pack8(x)
    return sp.Rows8(dev(q).view(torch.float8_e4m3fn), dev(e), cols), ow.unpack8(q, e)


def _check_product(got, a, b, log, dtype):
    P = a.shape[1]
    ref, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    err = P * 2.0 ** -23 * mag
    half = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps  # last place of zero
    with np.errstate(all="ignore"):
        if log:
            rel = err / ref
            assert rel[ref > 0].max(initial=0) < 0.01
            want = np.log(ref)
            tol = 1.01 * rel + 2.0 ** -22 * (np.abs(want) + 1)
        else:
            want, tol = ref, err
        tol = tol + half * np.abs(want) + tiny
        most = torch.finfo(dtype).max
        inner = np.isfinite(want) & (np.abs(want) < most * (1 - half))
        assert np.all(np.abs(got - want)[inner] <= (tol * (1 + half))[inner]), \
            (np.abs(got - want) / tol)[inner].max()
    assert np.array_equal(np.isneginf(got), np.isneginf(want) | (want <= -most * (1 + half)))


@pytest.mark.parametrize("m,n,cols", [(1, 1, 1), (1, 17, 50), (16, 16, 128), (17, 33, 129),
                                      (3, 1000, 500), (130, 257, 300), (65, 129, 1000),
                                      (300, 700, 513), (2, 5000, 64), (33, 4097, 100),
                                      (200, 40, 1024), (1000, 3, 20)])
@pytest.mark.parametrize("type,log", [("f32", True), ("f32", False), ("f16", True),
                                      ("bf16", False)])
def test_product(state, m, n, cols, type, log):
    say(f"product {m} x {n} x {cols} {type} log={log}")
    rng = np.random.default_rng(m + 10 * n + 100 * cols)
    a8, a = _packed(rng, m, cols, 2.0)
    b8, b = _packed(rng, n, cols, 3.0)
    if type in ("f16",) and not log:
        pytest.skip("range")
    for pad, at in ((0, 0), (5, 3)):
        out, buf = framed(m, n, TYPES[type], ld=n + pad, at=at)
        sp.spdp_product8(state.h, a8, b8, out, log=log)
        _check_product(out.double().cpu().numpy(), a, b, log, TYPES[type])
        assert frame_kept(buf, out)


@pytest.mark.parametrize("m,n", [(5, 300), (150, 300)])
def test_product_signs_zero_rows_and_nan(state, m, n):
    say(f"product of mixed signs {m} x {n}")
    rng = np.random.default_rng(3)
    a8, a = _packed(rng, m, 200, 1.0, sign=True)
    b8, b = _packed(rng, n, 200, 1.0, sign=True)
    a8.q[1].zero_()
    a[1] = 0
    out = torch.empty((m, n), device="cuda")
    sp.spdp_product8(state.h, a8, b8, out)
    _check_product(out.double().cpu().numpy(), a, b, False, torch.float32)
    assert (out[1] == 0).all()
    sp.spdp_product8(state.h, a8, b8, out, log=True)
    got = out.cpu().numpy()
    assert np.isneginf(got[1]).all()
    ref = a @ b.T
    sure = np.abs(ref) > 256 * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    assert np.array_equal(np.isnan(got)[sure], (ref < 0)[sure])
    b8.q.view(torch.uint8)[2, 7] = 127  # NaN
    sp.spdp_product8(state.h, a8, b8, out)
    got = out.cpu().numpy()
    assert np.isnan(got[:, 2]).all() and np.isfinite(np.delete(got, 2, 1)).all()


def test_product_range_of_scales(state):
    """Scales from end to end of what fp32 sums hold; probabilities near 1 and far below."""
    say("product, far scales")
    rng = np.random.default_rng(4)
    a = np.abs(rng.normal(size=(20, 300))) + 0.1
    b = np.abs(rng.normal(size=(40, 300))) + 0.1
    a[0] *= 1e30
    a[1, :128] *= 1e-30
    a[2] *= 1e-30
    b[3] *= 1e-8
    b[4, 128:] *= 1e-30
    a[5], b[5] = 0, 0
    a[5, 0] = b[5, 0] = 1.0
    (qa, ea), (qb, eb) = ow.pack8(a), ow.pack8(b)
    a8 = sp.Rows8(dev(qa).view(torch.float8_e4m3fn), dev(ea), 300)
    b8 = sp.Rows8(dev(qb).view(torch.float8_e4m3fn), dev(eb), 300)
    out = torch.empty((20, 40), device="cuda")
    for log in (False, True):
        sp.spdp_product8(state.h, a8, b8, out, log=log)
        _check_product(out.double().cpu().numpy(), ow.unpack8(qa, ea), ow.unpack8(qb, eb), log,
                       torch.float32)


def test_product_empty(state):
    say("product without rows")
    a, b = sp.Rows8.empty(0, 5), sp.Rows8.empty(3, 5)
    sp.spdp_product8(state.h, a, b, torch.empty((0, 3), device="cuda"))
    sp.spdp_product8(state.h, b, a, torch.empty((3, 0), device="cuda"))


# ---------------------------------------------------------------------------
# rules
# ---------------------------------------------------------------------------
def _scores(rng, rows, V, dtype, coarse=False):
    x = rng.normal(size=(rows, V)) * 3 - 4
    if coarse:
        x = np.round(x)
    return dev(x, dtype)


class RuleSet:
    """Rules for the library and the same for the oracle."""

    def __init__(self, rng, rows, V, listed=True, bias=True, mask=True, shared=False):
        kw, self.o = {}, {}
        if listed:
            docs = [rng.integers(-3, V + 3, size=[0, 1, 30, 200][i % 4]) for i in range(rows)]
            for i, d in enumerate(docs):
                if len(d) > 4:
                    d[:4] = i % V  # a word several times
            pen = np.stack([1 + rng.random(rows), rng.random(rows), rng.random(rows)], 1)
            kw.update(doc_off=dev(np.cumsum([0] + [len(d) for d in docs])),
                      words=dev(np.concatenate(docs).astype(np.int32)),
                      penalties=dev(pen, torch.float32))
            self.o.update(listed=docs, penalties=pen.astype(np.float32))
        if bias:
            t = rng.normal(size=(3, V)).astype(np.float32)
            of = np.zeros(rows, int) if shared else rng.integers(-1, 3, size=rows)
            kw.update(bias=dev(t), bias_of=None if shared else dev(of, torch.int32))
            self.o["bias"] = np.where(of[:, None] >= 0, t[np.maximum(of, 0)], 0)
            # (adding 0 changes nothing but a -0)
        if mask:
            t = rng.random((4, V)) < 0.6
            t[2] = False
            of = np.zeros(rows, int) if shared else rng.integers(-1, 4, size=rows)
            bits = np.zeros((4, -(-V // 32) * 32), np.uint8)
            bits[:, :V] = t
            bits[:, V:] = 1  # bits behind the last word mean nothing
            kw.update(mask=dev(np.packbits(bits, axis=1, bitorder="little").view("<i4").copy()),
                      mask_of=None if shared else dev(of, torch.int32))
            self.o["allowed"] = np.where(of[:, None] >= 0, t[np.maximum(of, 0)], True)
        self.c = sp.Rules(rows, V, **kw)

    def oracle(self, x):
        return ow.adjusted(x.float().cpu().numpy(), **self.o)


SIZES = [(1, 1), (2, 5), (1, 33), (7, 1000), (3, 4095), (2, 4097), (9, 10007), (130, 70)]


@pytest.mark.parametrize("rows,V", SIZES)
@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
def test_adjust(state, rows, V, type):
    say(f"adjust {rows} x {V} {type}")
    rng = np.random.default_rng(rows + V)
    for parts in ((1, 1, 1, 0), (1, 0, 0, 0), (0, 1, 0, 1), (0, 0, 1, 1), (0, 0, 1, 0),
                  (0, 0, 0, 0)):
        r = RuleSet(rng, rows, V, *(bool(p) for p in parts))
        for pad, at in ((0, 0), (3, 1)):
            x, xbuf = framed(rows, V, TYPES[type], ld=V + pad, at=at)
            x.copy_(_scores(rng, rows, V, TYPES[type]))
            want = torch.from_numpy(r.oracle(x)).to(TYPES[type])
            y, ybuf = framed(rows, V, TYPES[type], ld=V + 2 * pad, at=2 * at)
            before = xbuf.clone()
            sp.spdp_adjust(state.h, x, r.c, y)
            torch.testing.assert_close(y.cpu(), want, rtol=0, atol=0)
            assert frame_kept(ybuf, y) and torch.equal(before, xbuf)
            sp.spdp_adjust(state.h, x, r.c, x)  # in place
            torch.testing.assert_close(x.cpu(), want, rtol=0, atol=0)
            assert frame_kept(xbuf, x)


def test_adjust_scores_without_a_number(state):
    say("adjust: infinities, NaN, lowest values, masked and not")
    for type in ("f32", "f16", "bf16"):
        big = torch.finfo(TYPES[type]).max
        row = [np.nan, np.inf, -np.inf, -big, big, 0.0, -0.0, 1.0]
        x = dev(np.array([row, row, row]), TYPES[type])
        rng = np.random.default_rng(0)
        r = RuleSet(rng, 3, 8, listed=False, bias=False, mask=False)
        mask = dev(np.array([[0], [0xFF], [0b10101010]], np.int32))
        pen = dev(np.array([[2.0, 1.0, 0.5]] * 3, np.float32))
        r = sp.Rules(3, 8, mask=mask, mask_of=dev(np.arange(3, dtype=np.int32)), penalties=pen,
                     doc_off=dev(np.array([0, 8, 16, 24])),
                     words=dev(np.tile(np.arange(8), 3).astype(np.int32)))
        got = sp.spdp_adjust(state.h, x, r, torch.empty_like(x)).cpu()
        allowed = np.array([[0] * 8, [1] * 8, [0, 1] * 4], bool)
        want = torch.from_numpy(ow.adjusted(x.float().cpu().numpy(), [range(8)] * 3,
                                            [[2.0, 1.0, 0.5]] * 3, None, allowed)).to(TYPES[type])
        torch.testing.assert_close(got, want, rtol=0, atol=0, equal_nan=True)
        assert torch.isneginf(got[0]).all()


def test_rules_out_of_range(state):
    """Indices past their tables make the row NaN; offsets are clamped; nothing out of the
    arrays is read."""
    say("rules out of range")
    V = 50
    x = torch.zeros((6, V), device="cuda")
    bias = torch.ones((2, V), device="cuda")
    mask = dev(np.full((2, 2), -1, np.int32))
    of = dev(np.array([0, 1, 2, -1, -5, 2 ** 31 - 1], np.int32))
    for kw in (dict(bias=bias, bias_of=of), dict(mask=mask, mask_of=of)):
        y = sp.spdp_adjust(state.h, x, sp.Rules(6, V, **kw), torch.empty_like(x))
        assert torch.isnan(y).all(1).tolist() == [False, False, True, False, False, True]
        word, value = torch.empty((6, 2), dtype=torch.int32, device="cuda"), \
            torch.empty((6, 2), device="cuda")
        sp.spdp_top(state.h, x, word, value, work_for(6, V, 2), rules=sp.Rules(6, V, **kw))
        assert word[2].tolist() == [-1, -1] and word[0].tolist() == [0, 1]
        sp.spdp_draw(state.h, x, word, value, work_for(6, V), rules=sp.Rules(6, V, **kw))
        assert (word[5] == -1).all() and torch.isnan(value[5]).all() and (word[0] >= 0).all()
    off = dev(np.array([-7, 2, 1, 3, 99, 2 ** 40, 4]))
    words = dev(np.array([0, 1, 2, 3], np.int32))
    pen = dev(np.tile(np.array([1.0, 1.0, 0.0], np.float32), (6, 1)))
    r = sp.Rules(6, V, doc_off=off, words=words, penalties=pen)
    y = sp.spdp_adjust(state.h, x, r, torch.empty_like(x)).cpu().numpy()
    lists = [[0, 1], [], [1, 2], [3], [], []]
    want = np.zeros((6, V))
    for i, w in enumerate(lists):
        want[i, w] = -1
    np.testing.assert_array_equal(y, want)


def test_long_lists(state):
    """A document longer than its vocabulary, and counts beyond 16 bits."""
    say("adjust with 200 000 listed words")
    rng = np.random.default_rng(5)
    V = 5000
    docs = [np.full(150000, 4097), rng.integers(0, V, 50000)]
    pen = np.array([[1.5, 0.25, 2.0 ** -10]] * 2, np.float32)
    x = _scores(rng, 2, V, torch.float32)
    r = sp.Rules(2, V, doc_off=dev(np.array([0, 150000, 200000])),
                 words=dev(np.concatenate(docs).astype(np.int32)), penalties=dev(pen))
    y = sp.spdp_adjust(state.h, x, r, torch.empty_like(x)).cpu().numpy()
    np.testing.assert_array_equal(y, ow.adjusted(x.cpu().numpy(), docs, pen))


# ---------------------------------------------------------------------------
# best words
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("rows,V", SIZES + [(40, 20000)])
@pytest.mark.parametrize("k", [1, 7, 64, 256])
@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_top(state, rows, V, k, type):
    say(f"top {k} of {rows} x {V} {type}")
    rng = np.random.default_rng(rows + V + k)
    for coarse in (False, True):  # many ties
        x, _ = framed(rows, V, TYPES[type], ld=V + 3, at=1)
        x.copy_(_scores(rng, rows, V, TYPES[type], coarse))
        for r in (None, RuleSet(rng, rows, V, bias=not coarse)):
            want = ow.top(x.float().cpu().numpy() if r is None else r.oracle(x), k)
            word, wbuf = framed(rows, k, torch.int32, fill=9)
            value, vbuf = framed(rows, k, torch.float32)
            sp.spdp_top(state.h, x, word, value, work_for(rows, V, k), rules=r and r.c)
            np.testing.assert_array_equal(word.cpu().numpy(), want[0])
            np.testing.assert_array_equal(value.cpu().numpy(), want[1])
            assert frame_kept(wbuf, word, 9) and frame_kept(vbuf, value)


@pytest.mark.parametrize("V", [9, 300, 9000])
def test_top_special_rows(state, V):
    say(f"top: rows of one value, sorted rows, infinities, {V} words")
    x = np.zeros((9, V), np.float32)
    x[1] = np.arange(V)
    x[2] = -np.arange(V)
    x[3] = -np.inf
    x[4] = np.nan
    x[5, ::2] = -0.0  # ties with 0
    x[6, V // 2:] = np.inf
    x[7] = -np.inf
    x[7, V - 1] = -3.0e38
    x[8] = np.nan
    x[8, V // 2] = -np.inf
    x[8, V - 2] = -1
    for k in (1, 5, 256):
        want = ow.top(x, k)
        word = torch.empty((9, k), dtype=torch.int32, device="cuda")
        value = torch.empty((9, k), device="cuda")
        sp.spdp_top(state.h, dev(x), word, value, work_for(9, V, k))
        np.testing.assert_array_equal(word.cpu().numpy(), want[0])
        np.testing.assert_array_equal(value.cpu().numpy(), want[1])


# ---------------------------------------------------------------------------
# draws
# ---------------------------------------------------------------------------
def _check_draws(word, logp, x, u, temperature, most_skipped=0.01):
    ww, wl, gap = ow.drawn(x, u, temperature)
    sure = ~(gap <= 1e-11)
    assert (~sure).mean() <= most_skipped, (~sure).sum()
    np.testing.assert_array_equal(word[sure], ww[sure])
    law = ww >= 0
    assert np.array_equal(np.isnan(logp), ~law)
    # one rounding to fp32 of a logarithm whose fp64 error is far below it
    ok = sure & law
    assert np.all(np.abs(logp - wl)[ok] <= 2.0 ** -24 * 1.001 * np.abs(wl)[ok] + 1e-12)


@pytest.mark.parametrize("rows,V", SIZES + [(3, 100000)])
@pytest.mark.parametrize("n", [1, 5, 300])
@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_draw(state, rows, V, n, type):
    say(f"draw {n} of {rows} x {V} {type}")
    rng = np.random.default_rng(rows + V + n)
    for r, temperature in ((None, 1.0), (True, 1.0), (None, 0.25), (True, 3.0)):
        x, _ = framed(rows, V, TYPES[type], ld=V + 3, at=1)
        x.copy_(_scores(rng, rows, V, TYPES[type]))
        r = r and RuleSet(rng, rows, V)
        u = rng.random((rows, n))
        u[0, 0] = 0.0
        word, wbuf = framed(rows, n, torch.int32, fill=9)
        logp, lbuf = framed(rows, n, torch.float32)
        sp.spdp_draw(state.h, x, word, logp, work_for(rows, V), u=dev(u), rules=r and r.c,
                     temperature=temperature)
        xo = x.float().cpu().numpy() if r is None else r.oracle(x)
        _check_draws(word.cpu().numpy(), logp.cpu().numpy(), xo, u, temperature)
        assert frame_kept(wbuf, word, 9) and frame_kept(lbuf, logp)


@pytest.mark.parametrize("V", [6, 5000, 9000])
def test_draw_special_rows(state, V):
    """Rows without a law, a single allowed word, weights that vanish in most places, and
    uniforms at and outside the ends."""
    say(f"draw: special rows, {V} words")
    x = np.zeros((9, V), np.float32)
    x[0] = -np.inf
    x[1, 3] = np.nan
    x[2, V - 1] = np.inf
    x[3] = -np.inf
    x[3, V - 2] = -1e30                 # the only word
    x[4] = -800.0 * np.arange(V)        # all weight on word 0
    x[5] = -800.0 * np.arange(V)[::-1]  # all weight on the last word
    x[6, V // 2:] = -740.0              # weights near the smallest fp64
    x[7] = -3.0e38
    x[8, ::2] = -np.inf
    u = np.tile(np.array([0.0, 0.3, 1 - 2.0 ** -53, 1.0, 2.0, -1.0, np.nan, np.inf]), (9, 1))
    word = torch.empty((9, 8), dtype=torch.int32, device="cuda")
    logp = torch.empty((9, 8), device="cuda")
    sp.spdp_draw(state.h, dev(x), word, logp, work_for(9, V), u=dev(u))
    got = word.cpu().numpy()
    ww, wl, _ = ow.drawn(x, u)
    # the last word with weight is where 1 - 2^-53 may fall too, or the one before a border
    np.testing.assert_array_equal(np.delete(got, 2, 1), np.delete(ww, 2, 1))
    assert np.all((got[:, 2] >= 0) == (ww[:, 2] >= 0)) and np.all(got[3] == V - 2)
    assert np.array_equal(np.isnan(logp.cpu().numpy()), ww < 0)
    assert (got[:3] == -1).all() and (got[4] == 0).all() and (got[5] == V - 1).all()
    assert (got[8] % 2 == 1).all()


@pytest.mark.parametrize("V", [5000, 9000])
@pytest.mark.parametrize("lens", [(1535, 1536, 1537, 0), (1, 20000, 4096, 1540)])
def test_draw_from_long_documents(state, V, lens):
    """Documents around and beyond the length that a table of their words holds, with one word
    in half of a document's places and penalties that a wrong count would show."""
    say(f"draw: documents of {lens} words of {V}")
    rng = np.random.default_rng(V + lens[0])
    rows, n = len(lens), 200
    docs = [rng.integers(-3, V + 3, size=m) for m in lens]
    for i, d in enumerate(docs):
        d[: len(d) // 2] = V - 1 - i
    pen = np.stack([1 + rng.random(rows), rng.random(rows), 2.0 ** -9 * rng.random(rows)], 1)
    pen = pen.astype(np.float32)
    x = _scores(rng, rows, V, torch.float32)
    for i in range(rows):
        x[i, V - 20:] += 6  # (the counted word and its neighbours are drawn often)
    u = rng.random((rows, n))
    r = sp.Rules(rows, V, doc_off=dev(np.cumsum([0] + list(lens))),
                 words=dev(np.concatenate(docs).astype(np.int32)), penalties=dev(pen))
    word = torch.empty((rows, n), dtype=torch.int32, device="cuda")
    logp = torch.empty((rows, n), device="cuda")
    sp.spdp_draw(state.h, x, word, logp, work_for(rows, V), u=dev(u), rules=r)
    _check_draws(word.cpu().numpy(), logp.cpu().numpy(),
                 ow.adjusted(x.cpu().numpy(), docs, pen), u, 1.0)


@pytest.mark.parametrize("rows,n", [(1, 384), (1, 385), (2, 5000), (255, 400), (256, 400)])
def test_many_draws(state, rows, n):
    """Draws of rows of one chunk, by the row's own workgroup or by several."""
    say(f"draw {n} of {rows} x 3000")
    rng = np.random.default_rng(rows + n)
    V = 3000
    x = _scores(rng, rows, V, torch.float32)
    r = RuleSet(rng, rows, V)
    u = rng.random((rows, n))
    u[0, 7] = 1.0
    word, wbuf = framed(rows, n, torch.int32, fill=9)
    logp, lbuf = framed(rows, n, torch.float32)
    sp.spdp_draw(state.h, x, word, logp, work_for(rows, V), u=dev(u), rules=r.c)
    some = np.r_[0:min(rows, 3), rows - min(rows, 3):rows]
    xo = r.oracle(x)
    last = np.flatnonzero(xo[0] > -np.inf)
    assert word[0, 7].item() == (last[-1] if len(last) else -1)
    word[0, 7], logp[0, 7] = word[0, 8].clone(), logp[0, 8].clone()
    u[0, 7] = u[0, 8]
    _check_draws(word[dev(some)].cpu().numpy(), logp[dev(some)].cpu().numpy(), xo[some], u[some], 1.0)
    assert frame_kept(wbuf, word, 9) and frame_kept(lbuf, logp)


def test_draws_do_not_depend_on_their_company(state):
    """The same uniforms draw the same words alone, with others and in other batches of rows."""
    say("draw: alone and together")
    rng = np.random.default_rng(77)
    for V in (3000, 30000):
        rows, n = 300, 1000
        x = _scores(rng, rows, V, torch.bfloat16)
        u = dev(rng.random((rows, n)))
        word, logp = _outs(rows, n)
        sp.spdp_draw(state.h, x, word, logp, work_for(rows, V), u=u)
        for i, j, k in ((0, 1, 1000), (0, 1, 384), (5, 6, 1), (10, 40, 70), (0, 255, 999)):
            w, p = _outs(j - i, k)
            sp.spdp_draw(state.h, x[i:j], w, p, work_for(j - i, V), u=u[i:j, :k].contiguous())
            assert torch.equal(w, word[i:j, :k]) and torch.equal(p, logp[i:j, :k]), (V, i, j, k)


def test_draw_of_many_chunks(state):
    """More chunks than a wavefront has lanes, some of them without weight, the last among
    them, and more draws than it makes at a time."""
    say("draw: 1 200 000 words")
    rng = np.random.default_rng(12)
    rows, V, n = 3, 1200000, 150
    x = _scores(rng, rows, V, torch.float32)
    x[0, 700000:] = -np.inf
    x[1, : 600000] = -np.inf
    x[2, 8192 * 64: 8192 * 128] = -np.inf
    u = rng.random((rows, n))
    u[:, 0] = 0.0
    u[:, 77] = 1.0
    u[:, 149] = np.nan
    word = torch.empty((rows, n), dtype=torch.int32, device="cuda")
    logp = torch.empty((rows, n), device="cuda")
    sp.spdp_draw(state.h, x, word, logp, work_for(rows, V), u=dev(u))
    word, logp = word.cpu().numpy(), logp.cpu().numpy()
    ends = [699999, V - 1, V - 1]
    np.testing.assert_array_equal(word[:, 77], ends)
    np.testing.assert_array_equal(word[:, 149], ends)
    keep = [i for i in range(n) if i not in (77, 149)]
    _check_draws(word[:, keep], logp[:, keep], x.cpu().numpy(), u[:, keep], 1.0)


def test_draw_by_seed(state):
    say("draw by seed")
    rng = np.random.default_rng(8)
    rows, V, n, seed, step = 5, 3000, 40, 0x123456789ABCDEF, 7
    x = _scores(rng, rows, V, torch.float32)
    word = torch.empty((rows, n), dtype=torch.int32, device="cuda")
    logp = torch.empty((rows, n), device="cuda")
    sp.spdp_draw(state.h, x, word, logp, work_for(rows, V), seed=seed, step=step)
    u = np.array([oracle.philox_word0(seed, i, step, 4) for i in range(rows * n)])
    _check_draws(word.cpu().numpy(), logp.cpu().numpy(), x.cpu().numpy(),
                 u.reshape(rows, n) * 2.0 ** -32, 1.0)


def test_no_rows_and_no_draws(state):
    say("top and draw of nothing")
    x = torch.empty((0, 50), device="cuda")
    e = lambda *s, dtype: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    w = work_for(0, 50, 3)
    sp.spdp_top(state.h, x, e(0, 3, dtype=torch.int32), e(0, 3, dtype=torch.float32), w)
    sp.spdp_draw(state.h, x, e(0, 3, dtype=torch.int32), e(0, 3, dtype=torch.float32), w)
    x = torch.zeros((2, 50), device="cuda")
    sp.spdp_draw(state.h, x, e(2, 0, dtype=torch.int32), e(2, 0, dtype=torch.float32),
                 work_for(2, 50))
    sp.spdp_adjust(state.h, e(0, 50, dtype=torch.float32), sp.Rules(0, 50),
                   e(0, 50, dtype=torch.float32))


@pytest.mark.parametrize("type", ["f32", "f16"])
def test_long_rows(state, type):
    """Rows of more chunks than a wavefront has lanes, with rules."""
    V, n, k = 1200001, 64, 200
    say(f"top and draw of 2 x {V} {type}")
    rng = np.random.default_rng(21)
    x = _scores(rng, 2, V, TYPES[type])
    x[1, :700000] = -np.inf
    mask = np.full((1, -(-V // 32)), 0x5DB5D5B7, np.uint32)
    docs = [rng.integers(0, V, 3000), np.array([5, V - 1, V - 1])]
    pen = np.array([[1.5, 0.5, 0.25]] * 2, np.float32)
    r = sp.Rules(2, V, doc_off=dev(np.array([0, 3000, 3003])),
                 words=dev(np.concatenate(docs).astype(np.int32)), penalties=dev(pen),
                 mask=dev(mask.view(np.int32)))
    allowed = np.unpackbits(mask.view(np.uint8), axis=1, bitorder="little")[:, :V].astype(bool)
    xo = ow.adjusted(x.float().cpu().numpy(), docs, pen, None, np.repeat(allowed, 2, 0))
    word = torch.empty((2, k), dtype=torch.int32, device="cuda")
    value = torch.empty((2, k), device="cuda")
    sp.spdp_top(state.h, x, word, value, work_for(2, V, k), rules=r)
    order = [np.lexsort((np.arange(V), -row.astype(np.float64)))[:k] for row in xo]
    np.testing.assert_array_equal(word.cpu().numpy(), order)
    np.testing.assert_array_equal(value.cpu().numpy(), np.take_along_axis(xo, np.array(order), 1))
    u = rng.random((2, n))
    u[:, 0], u[:, 1] = 1.0, 0.0
    word = torch.empty((2, n), dtype=torch.int32, device="cuda")
    logp = torch.empty((2, n), device="cuda")
    sp.spdp_draw(state.h, x, word, logp, work_for(2, V), u=dev(u), rules=r)
    _check_draws(word.cpu().numpy(), logp.cpu().numpy(), xo, u, 1.0)


@pytest.mark.parametrize("m,n", [(3, 100), (70, 200)])
def test_product_many_columns(state, m, n):
    """More columns than the documents' tile holds at a time."""
    say(f"product {m} x {n} x 5000")
    rng = np.random.default_rng(22)
    a8, a = _packed(rng, m, 5000, 1.0)
    b8, b = _packed(rng, n, 5000, 1.0)
    for log in (False, True):
        out = torch.empty((m, n), device="cuda")
        sp.spdp_product8(state.h, a8, b8, out, log=log)
        _check_product(out.double().cpu().numpy(), a, b, log, torch.float32)


@pytest.mark.parametrize("n", [63, 64, 1000])
def test_product_does_not_depend_on_the_batch(state, n):
    say(f"product: rows alone and together, {n} words")
    rng = np.random.default_rng(23)
    a8, _ = _packed(rng, 300, 700, 2.0)
    b8, _ = _packed(rng, n, 700, 2.0)
    whole = sp.spdp_product8(state.h, a8, b8, torch.empty((300, n), device="cuda"), log=True)
    for i, j in ((0, 1), (5, 6), (0, 16), (3, 20), (0, 40), (100, 164), (7, 97), (11, 300)):
        part = sp.Rows8(a8.q[i:j], a8.e[i:j], 700)
        out = torch.empty((j - i, n), device="cuda")
        assert torch.equal(sp.spdp_product8(state.h, part, b8, out, log=True), whole[i:j]), (i, j)


@pytest.mark.parametrize("m", [1, 6, 60, 300])
def test_product_in_16_bits_is_the_rounded_one(state, m):
    """In every kernel: fp32 first, then the output's type, with nothing rounded in between."""
    say(f"product: {m} documents in 16 bits")
    rng = np.random.default_rng(m)
    theta, phi = rng.dirichlet(np.full(8, 0.1), size=m), rng.random((100001, 8)) ** 8 + 1e-9
    a, b = (sp.spdp_pack8(state.h, dev(x), sp.Rows8.empty(*x.shape)) for x in (theta, phi))
    for log in (False, True):
        want = sp.spdp_product8(state.h, a, b, torch.empty((m, 100001), device="cuda"), log=log)
        for t in (torch.float16, torch.bfloat16):
            got = torch.empty((m, 100001), dtype=t, device="cuda")
            assert torch.equal(sp.spdp_product8(state.h, a, b, got, log=log), want.to(t)), (t, log)


# ---------------------------------------------------------------------------
# refusals that need a device
# ---------------------------------------------------------------------------
def test_refusals_on_device(state):
    say("refusals on the device")
    x = torch.zeros((4, 100), device="cuda")
    word = torch.empty((4, 3), dtype=torch.int32, device="cuda")
    value = torch.empty((4, 3), device="cuda")

    def refused(text, call, *a, **kw):
        with pytest.raises(sp.SpdpError) as e:
            call(*a, **kw)
        assert e.value.code == sp.SPDP_E_ARG and text in str(e.value), str(e.value)

    r = sp.Rules(4, 100)
    both = torch.zeros(1000, device="cuda")
    refused("overlap", sp.spdp_adjust, state.h, both[:400].view(4, 100), r,
            both[100:500].view(4, 100))
    refused("a workspace of", sp.spdp_top, state.h, x, word, value,
            torch.empty(16, dtype=torch.uint8, device="cuda"))
    refused("a workspace of", sp.spdp_draw, state.h, x, word, value, None)
    refused("aligned", sp.spdp_draw, state.h, x, word, value,
            torch.empty(1 << 16, dtype=torch.uint8, device="cuda")[8:])
    refused("rules for 3 x 100", sp.spdp_top, state.h, x, word, value, work_for(4, 100, 3),
            rules=sp.Rules(3, 100))
    refused("need doc_off", sp.spdp_adjust, state.h, x,
            sp.Rules(4, 100, penalties=torch.ones((4, 3), device="cuda")), x)
    refused("without penalties", sp.spdp_adjust, state.h, x, sp.Rules(
        4, 100, doc_off=torch.zeros(5, dtype=torch.int64, device="cuda"),
        words=torch.zeros(1, dtype=torch.int32, device="cuda")), x)
    refused("without its table", sp.spdp_adjust, state.h, x, sp.Rules(
        4, 100, mask_of=torch.zeros(4, dtype=torch.int32, device="cuda")), x)
    with pytest.raises(ValueError):  # (torch has no address for it)
        sp.Rules(4, 100, bias=x[:0])
    L = sp.lib()
    none = sp._Rules(rows=4, n_words=100, bias=x.data_ptr())
    assert L.spdp_adjust(state.h, x.data_ptr(), 100, x.data_ptr(), 100, sp.SPDP_F32,
                         ctypes.addressof(none)) == sp.SPDP_E_ARG
    assert "rules: bias has no rows" in sp.spdp_last_error()
    # misaligned arrays of the rules
    off = torch.zeros(64, dtype=torch.int32, device="cuda")
    for field in ("doc_off", "words", "penalties", "bias", "mask"):
        c = sp._Rules(rows=4, n_words=100, n_bias=1, n_masks=1, n_listed=4)
        if field in ("doc_off", "words", "penalties"):
            for f in ("doc_off", "words", "penalties"):
                setattr(c, f, x.data_ptr())
        setattr(c, field, off.data_ptr() + 2)
        assert L.spdp_adjust(state.h, x.data_ptr(), 100, x.data_ptr(), 100, sp.SPDP_F32,
                             ctypes.addressof(c)) == sp.SPDP_E_ARG
        assert f"{field} is misaligned" in sp.spdp_last_error()
    host = np.zeros((4, 100), np.float32)
    assert L.spdp_adjust(state.h, host.ctypes.data, 100, x.data_ptr(), 100, sp.SPDP_F32,
                         r.ref) == sp.SPDP_E_ARG and "x is not device" in sp.spdp_last_error()
    # rows far past the allocation
    big = sp._Rules(rows=1 << 30, n_words=100)
    assert L.spdp_adjust(state.h, x.data_ptr(), 100, x.data_ptr(), 100, sp.SPDP_F32,
                         ctypes.addressof(big)) == sp.SPDP_E_ARG
    assert "run past its allocation" in sp.spdp_last_error()


# ---------------------------------------------------------------------------
# all of them
# ---------------------------------------------------------------------------
def _model(rng, D, V, K):
    theta = rng.dirichlet(np.full(K, 0.1), size=D)
    phi = rng.dirichlet(np.full(V, 0.05), size=K).T + 1e-9
    out = []
    for x in (theta, phi):
        q, e = ow.pack8(x)
        out.append(sp.Rows8(dev(q).view(torch.float8_e4m3fn), dev(e), K))
    return out


def _outs(D, n):
    return (torch.full((D, n), -7, dtype=torch.int32, device="cuda"),
            torch.full((D, n), 7.0, device="cuda"))


@pytest.mark.parametrize("D,V,K", [(1, 500, 10), (37, 5001, 50), (130, 9000, 200)])
def test_predict_is_its_steps(state, D, V, K):
    say(f"predict {D} x {V} x {K}")
    rng = np.random.default_rng(D + V)
    docs, words = _model(rng, D, V, K)
    r = RuleSet(rng, D, V)
    u = dev(rng.random((D, 9)))
    for type in ("f32", "bf16"):
        t = TYPES[type]
        scores = torch.empty((D, V), dtype=t, device="cuda")
        sp.spdp_product8(state.h, docs, words, scores, log=True)
        want_top, want_drawn = _outs(D, 20), _outs(D, 9)
        sp.spdp_top(state.h, scores, *want_top, work_for(D, V, 20), rules=r.c)
        sp.spdp_draw(state.h, scores, *want_drawn, work_for(D, V), u=u, rules=r.c)
        # with room for all documents, for one, and for some
        full = sp.spdp_predict_work(D, V, t, 20)
        one = -(-V * scores.element_size() // 256) * 256 + sp.spdp_words_work(1, V, 20)
        for room in {full, one, min(full, 5 * one + 100)}:
            top, drawn = _outs(D, 20), _outs(D, 9)
            work = torch.empty(room, dtype=torch.uint8, device="cuda")
            sp.spdp_predict(state.h, docs, words, work, rules=r.c, dtype=t, top=top, drawn=drawn,
                            u=u)
            for a, b in zip(top + drawn, want_top + want_drawn):
                assert torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0))
        with pytest.raises(sp.SpdpError):
            sp.spdp_predict(state.h, docs, words, work[:one - 256], rules=r.c, dtype=t, top=top)
        # the scores are kept: adjusted, and the words come from them
        sp.spdp_adjust(state.h, scores, r.c, scores)
        kept, buf = framed(D, V, t, ld=V + 5, at=3)
        top = _outs(D, 20)
        sp.spdp_predict(state.h, docs, words, work_for(D, V, 20), rules=r.c, scores=kept, top=top)
        assert torch.equal(kept, scores) and frame_kept(buf, kept)
        want = _outs(D, 20)
        sp.spdp_top(state.h, scores, *want, work_for(D, V, 20))
        for a, b in zip(top, want):
            assert torch.equal(a, b)
        if type == "f32":
            for a, b in zip(top, want_top):
                assert torch.equal(a, b)
    # seeded draws do not depend on how many documents are held at a time
    drawn = [_outs(D, 3) for _ in range(2)]
    for d, room in zip(drawn, (sp.spdp_predict_work(D, V, t), one)):
        sp.spdp_predict(state.h, docs, words, torch.empty(room, dtype=torch.uint8, device="cuda"),
                        dtype=t, drawn=d, seed=5, step=1)
    assert all(torch.equal(a, b) for a, b in zip(*drawn))


def test_predict_of_a_trained_state():
    """From counts to words: estimates, 8-bit rows, scores, rules, words, against the
    oracle on the estimates themselves."""
    say("words of a trained state")
    wl = synth.workload(0)
    cp = synth.generate(wl, 0)
    s = sp.Sampler(cp.words, cp.doc_off, cp.doc_group, cp.n_groups, cp.vocab, wl.K, wl.alpha,
                   wl.a, wl.b, wl.gamma)
    for sweep in range(20):
        s.sweep(sweep, 3)
    theta, _, phi = s.estimates(0, 1)
    docs = [d for d in range(len(cp.doc_group)) if cp.doc_group[d] == 0][:40]
    lists = [cp.words[cp.doc_off[d]:cp.doc_off[d + 1]] for d in docs]
    allowed = np.ones(cp.vocab, bool)
    allowed[::7] = False
    word, value, dw, dl = s.predict(theta[docs], phi[0], top=10, draws=200, seed=11,
                                    doc_words=lists, penalties=(1.0, 50.0, 0.0), allowed=allowed)
    exact = np.log(theta[docs] @ phi[0].T)
    # a value in 8 bits is off by 2^-4 at most (or 2^-10 of its block's scale, far below
    # the sums here), a product of two by (1 + 2^-4)^2, its logarithm by 0.13
    for i, w in enumerate(lists):
        seen = np.isin(np.arange(cp.vocab), w)
        want = np.where(allowed, exact[i] - 50.0 * seen, -np.inf)
        assert np.all(np.abs(value[i] - want[word[i]]) <= 0.13)
        assert not np.isin(word[i], w).any() and allowed[word[i]].all()
        best = np.sort(want)[::-1][:10]
        assert np.all(np.abs(value[i] - best) <= 0.13)
        assert allowed[dw[i]].all() and not np.isin(dw[i], w).any()
    again = s.predict(theta[docs], phi[0], draws=200, seed=11, doc_words=lists,
                      penalties=(1.0, 50.0, 0.0), allowed=allowed)
    assert np.array_equal(again[2], dw) and again[0].shape == (40, 0)
    assert s.check() == 0
    s.close()


def test_predict_without_a_tensor_library():
    """In a program that has loaded the library only, whose HIP runtime is not torch's."""
    say("predict in a process of its own")
    code = """
import sys
import numpy as np
from paper_1510_06549_amd import spdp as sp
s = sp.Sampler(np.array([0, 1], np.int32), np.array([0, 2], np.int64), np.array([0], np.int32),
               1, 2, 1, 0.1, 0.5, 1.0, 0.1)
s.sweep(0, 1)
rng = np.random.default_rng(0)
theta, phi = rng.random((3, 7)), rng.random((600, 7))
theta, phi = np.round(theta * 8 + 1), np.round(phi * 8 + 1)  # (exact in 8 bits)
word, value, drawn, logp = s.predict(theta, phi, top=5, draws=4, seed=3)
exact = theta @ phi.T
want = np.argsort(-exact, axis=1, kind='stable')[:, :5]
assert np.array_equal(word, want), (word, want)
assert np.allclose(np.exp(value), np.take_along_axis(exact, want, 1), rtol=1e-5)
assert drawn.shape == (3, 4) and (drawn >= 0).all() and (drawn < 600).all()
assert [x.shape for x in s.predict(theta[:0], phi, top=5)] == [(0, 5), (0, 5), (0, 0), (0, 0)]
s.close()
assert 'torch' not in sys.modules
print('ok')
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100,
                          cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stderr[-2000:]


@pytest.mark.parametrize("V", [5000, 20000])
def test_captured_and_on_streams(V):
    """A captured chain, replayed between eager calls with other inputs, and two states on
    streams of their own with workspaces of their own."""
    say("captured words")
    rng = np.random.default_rng(12)
    D, K = 20, 60
    stream = torch.cuda.Stream()
    s, e = _state(stream), _state()
    theta = [dev(rng.dirichlet(np.full(K, 0.2), size=D)) for _ in range(3)]
    _, words = _model(rng, 1, V, K)
    r = RuleSet(rng, D, V)
    u = dev(rng.random((D, 9)))

    def chain(h, x, packed, work, outs):
        sp.spdp_pack8(h, x, packed)
        sp.spdp_predict(h, packed, words, work, rules=r.c, top=outs[0], drawn=outs[1], u=u)
        sp.spdp_product8(h, packed, words, outs[2][0])
        sp.spdp_adjust(h, outs[2][0], r.c, outs[2][0])

    def room():
        return (sp.Rows8.empty(D, K), torch.empty(sp.spdp_predict_work(D, V, torch.float32, 20),
                                                  dtype=torch.uint8, device="cuda"),
                (_outs(D, 20), _outs(D, 9),
                 (torch.empty((D, V), dtype=torch.float16, device="cuda"),)))

    x = theta[0].clone()
    mine, other = room(), room()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        chain(s.h, x, *mine)
    for t in theta + theta[:1]:
        with torch.cuda.stream(stream):
            x.copy_(t)
            graph.replay()
        chain(e.h, t, *other)  # at the same time, on the null stream
        torch.cuda.synchronize()
        for a, b in zip(sum(mine[2], ()), sum(other[2], ())):
            assert torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0))
    s.close()
    e.close()


# ---------------------------------------------------------------------------
# more rows than a launch holds
# ---------------------------------------------------------------------------
LAUNCH = (1 << 23) - 1  # workgroups


def test_more_rows_than_a_launch_holds(state):
    say("adjust, top and draw of 2^23 + 9 rows of 3 words")
    rng = np.random.default_rng(31)
    rows, V, seed = LAUNCH + 10, 3, 77
    x = torch.empty((rows, V), dtype=torch.float16, device="cuda").normal_()
    bias = torch.tensor([[0.5, -0.25, 1.0], [2.0, 0.0, -1.0]], device="cuda")
    of = torch.randint(-1, 2, (rows,), dtype=torch.int32, device="cuda")
    r = sp.Rules(rows, V, bias=bias, bias_of=of)
    y = sp.spdp_adjust(state.h, x, r, torch.empty_like(x))
    add = torch.where(of[:, None] >= 0, bias[of.clamp(min=0).long()], torch.zeros((), device="cuda"))
    assert torch.equal(y, (x.float() + add).half())
    word = torch.empty((rows, 2), dtype=torch.int32, device="cuda")
    value = torch.empty((rows, 2), device="cuda")
    sp.spdp_top(state.h, x, word, value, work_for(rows, V, 2), rules=r)
    sample = np.r_[0:5, LAUNCH - 5:rows, rng.integers(0, rows, 500)]
    xs = (x.float() + add)[dev(sample)].cpu().numpy()
    want = ow.top(xs, 2)
    np.testing.assert_array_equal(word[dev(sample)].cpu().numpy(), want[0])
    np.testing.assert_array_equal(value[dev(sample)].cpu().numpy(), want[1])
    sp.spdp_draw(state.h, x, word, value, work_for(rows, V), rules=r, seed=seed, step=3)
    u = np.array([[oracle.philox_word0(seed, 2 * i + t, 3, 4) for t in range(2)]
                  for i in sample.tolist()]) * 2.0 ** -32
    _check_draws(word[dev(sample)].cpu().numpy(), value[dev(sample)].cpu().numpy(), xs, u, 1.0)


def test_more_packed_rows_than_a_launch_holds(state):
    say("pack of 2^26 rows and products of 2^24 and 2^28")
    rows = 8 * LAUNCH + 3
    x = torch.arange(rows, device="cuda", dtype=torch.int32).remainder_(16).float()[:, None]
    p = sp.spdp_pack8(state.h, x, sp.Rows8.empty(rows, 1))
    for i in range(0, rows, 1 << 24):
        q = p.q[i:i + (1 << 24), 0].float() * p.e[i:i + (1 << 24), 0].float().sub_(127).exp2_()
        assert torch.equal(q, x[i:i + (1 << 24), 0])  # (4 bits: exact)
    del p, x, q
    for m, n in (((1 << 24) + 5, 3), (2, (1 << 28) + 70)):
        sides = []
        for size in (m, n):
            q = torch.zeros((size, 128), dtype=torch.uint8, device="cuda")
            q[:, 0] = 0x38  # 1
            e = torch.full((size, 1), 127, dtype=torch.uint8, device="cuda")
            e[-1] = 128
            e[0] = 129
            sides.append((sp.Rows8(q.view(torch.float8_e4m3fn), e, 1),
                          e[:, 0].float().sub_(127).exp2_()))
        (a, fa), (b, fb) = sides
        c = torch.empty((m, n), dtype=torch.float16, device="cuda")
        sp.spdp_product8(state.h, a, b, c)
        assert torch.equal(c, (fa[:, None] * fb[None, :]).half())
        del sides, a, b, c, q, e, fa, fb


def test_smallest_scores(state):
    """Scores below the normal range of fp32 keep their order, next to zeros of both signs."""
    say("top of denormal scores")
    x = np.zeros((2, 9000), np.float32)
    x[0] = np.arange(9000) % 4500 * np.float32(1.4e-45)
    x[1] = -x[0]
    x[1, ::7] = 0.0
    for k in (1, 50, 256):
        word = torch.empty((2, k), dtype=torch.int32, device="cuda")
        value = torch.empty((2, k), device="cuda")
        sp.spdp_top(state.h, dev(x), word, value, work_for(2, 9000, k))
        want = ow.top(x, k)
        np.testing.assert_array_equal(word.cpu().numpy(), want[0])
        np.testing.assert_array_equal(value.cpu().numpy(), want[1])


@pytest.mark.parametrize("k", [1, 3, 5, 200, 256])
def test_top_of_many_parts(state, k):
    """A row of more parts than a workgroup has threads, with ties and with parts that hold
    fewer than k words."""
    say(f"top {k} of 5 000 000 words")
    V = 5000000
    x = torch.empty((2, V), device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(k))
    x[0] = (x[0] * 8).round()  # (many ties)
    x[1, 100000:4900000] = -np.inf
    word = torch.empty((2, k), dtype=torch.int32, device="cuda")
    value = torch.empty((2, k), device="cuda")
    sp.spdp_top(state.h, x, word, value, work_for(2, V, k))
    for i, row in enumerate(x.cpu().numpy()):
        want = np.argsort(-row, kind="stable")[:k]
        np.testing.assert_array_equal(word[i].cpu().numpy(), want)
        np.testing.assert_array_equal(value[i].cpu().numpy(), row[want])


def test_more_scores_than_32_bits_count(state):
    """The last documents of 2.2e9 scores have the words that they have alone."""
    say("22 000 x 100 001 scores")
    rng = np.random.default_rng(9)
    D, V, K, tail = 22000, 100001, 8, 6
    assert D * V > 1 << 31
    docs, words = (sp.spdp_pack8(state.h, dev(x), sp.Rows8.empty(*x.shape)) for x in
                   (rng.dirichlet(np.full(K, 0.1), size=D), rng.dirichlet(np.full(V, 0.05), K).T + 1e-9))
    last = sp.Rows8(docs.q[-tail:].contiguous(), docs.e[-tail:].contiguous(), K)
    bias = torch.empty((1, V), device="cuda").normal_()
    few, all_ = (sp.Rules(n, V, bias=bias) for n in (tail, D))
    got, want = [], []
    for d, n, r, to in ((docs, D, all_, got), (last, tail, few, want)):
        x = torch.empty((n, V), dtype=torch.float16, device="cuda")
        sp.spdp_product8(state.h, d, words, x, log=True)
        sp.spdp_adjust(state.h, x, r, x)
        u = torch.full((n, 7), 0.6, dtype=torch.float64, device="cuda")
        u[:, 3] = 0.01
        w = work_for(n, V, 9)
        top, drawn = _outs(n, 9), _outs(n, 7)
        sp.spdp_top(state.h, x, *top, w)
        sp.spdp_draw(state.h, x, *drawn, w, u=u)
        to += [t[-tail:].clone() for t in (x, *top, *drawn)]
        del x
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (got[1] >= 0).all() and (got[3] >= 0).all()


def test_pack_every_power_of_two(state):
    """All of fp64 from its least value to its largest, alone in a block and beside 1: beyond
    448 2^127, the largest scale, there is no number."""
    say("pack, every power of two of fp64")
    two = np.ldexp(1.0, np.arange(-1074, 1024))
    x = np.concatenate([two, -1.75 * two[:-1], 2.0 ** 127 * np.array(
        [448.0, np.nextafter(448.0, 512.0), -448.0, -np.nextafter(448.0, 512.0)]),
        [1e160, -1e195, 1.5 * 2.0 ** 640, 1.75 * 2.0 ** 647, np.finfo(np.float64).max]])
    for beside in (False, True):
        rows = np.stack([x, np.ones_like(x)], 1) if beside else x[:, None]
        out = sp.Rows8.empty(*rows.shape)
        sp.spdp_pack8(state.h, dev(rows), out)
        q, e = ow.pack8(rows)
        np.testing.assert_array_equal(out.e.cpu().numpy(), e)
        np.testing.assert_array_equal(ow.value8(out.q.view(torch.uint8).cpu().numpy()),
                                      ow.value8(q))


@pytest.mark.parametrize("V,temperature", [(20000, 0.01), (20000, 1e-3), (70000, 0.004),
                                           (600000, 0.003), (5000, 0.01)])
def test_draw_ends_at_low_temperatures(state, V, temperature):
    """Uniforms at the ends draw the first and the last word with weight, where most words'
    weights are below the least fp64 value, beside the row's largest if not their chunk's."""
    say(f"draw: ends of {V} words at {temperature}")
    rng = np.random.default_rng(V)
    x = _scores(rng, 6, V, torch.float32)
    x[3:] *= 0.5
    u = np.tile(np.array([0.0, -1.0, 1.0, np.nan, 0.37, 0.99]), (6, 1))
    for r in (None, RuleSet(rng, 6, V, listed=False)):
        word, logp = _outs(6, 6)
        sp.spdp_draw(state.h, x, word, logp, work_for(6, V), u=dev(u), rules=r and r.c,
                     temperature=temperature)
        xo = x.cpu().numpy() if r is None else r.oracle(x)
        _check_draws(word.cpu().numpy(), logp.cpu().numpy(), xo, u, temperature, most_skipped=0.2)


def test_calls_after_a_failed_allocation(state):
    """What an allocation that failed leaves behind is no error of the next call."""
    say("calls after an allocation that failed")
    with pytest.raises(sp.SpdpError):
        sp._Device((1 << 50,), "uint8")
    out = sp.spdp_pack8(state.h, torch.ones((2, 3), device="cuda"), sp.Rows8.empty(2, 3))
    assert (out.q[:, :3].float() == 256).all()


def test_predict_words_beyond_32_bits(state):
    """Listed words that are none of the vocabulary's are ignored, however large."""
    say("predict: listed words beyond 32 bits")
    theta, phi = np.ones((2, 3)), np.arange(1, 31).reshape(10, 3) / 32.0
    plain = state.predict(theta, phi, top=4)[:2]
    odd = [np.array([2 ** 32 + 9, -1, 2 ** 40, 10]), [2 ** 33 + 8, -2 ** 31 - 1 + 9]]
    got = state.predict(theta, phi, top=4, doc_words=odd, penalties=(1.0, 1e9, 0.0))[:2]
    for a, b in zip(got, plain):
        np.testing.assert_array_equal(a, b)


# ---------------------------------------------------------------------------
# products of every shape of workgroup
# ---------------------------------------------------------------------------
def _model8(state, seed, m, n, cols):
    """Packed theta- and phi-like rows (positive, zeros among them, scales far apart) and their
    values in fp64, on the device."""
    gen = torch.Generator("cuda").manual_seed(seed)
    sides = []
    for rows, spread in ((m, 2.0), (n, 3.0)):
        x = torch.randn((rows, cols), device="cuda", generator=gen).mul_(spread).exp_()
        x[torch.rand((rows, cols), device="cuda", generator=gen) < 0.05] = 0
        x *= torch.randn((rows, 1), device="cuda", generator=gen).mul_(2).exp_()
        p = sp.spdp_pack8(state.h, x, sp.Rows8.empty(rows, cols))
        nb = p.e.shape[1]
        v = p.q.double().view(rows, nb, 128) * torch.exp2(p.e.double() - 127)[:, :, None]
        sides.append((p, v.view(rows, nb * 128)))
    return sides


def _all_products(state, m, n, cols, type, log, ld):
    """Every output within the sums' tolerance, and rows equal to those of batches of 16
    (which a kernel of their own makes)."""
    (a8, a), (b8, b) = _model8(state, m + n + cols, m, n, cols)
    dtype = TYPES[type]
    out, buf = framed(m, n, dtype, ld=ld, fill=-3.0)
    sp.spdp_product8(state.h, a8, b8, out, log=log)
    assert frame_kept(buf, out, -3.0)
    del buf
    # (sums of positive values: off by P 2^-23 of themselves at most)
    rel = a.shape[1] * 2.0 ** -23
    half = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    step = max(1, 50000000 // n)
    bt = b.T.contiguous()
    for i in range(0, m, step):
        ref = a[i:i + step] @ bt
        if log:
            want = ref.log()
            tol = 1.01 * rel + 2.0 ** -22 * (want.abs() + 1)
        else:
            want, tol = ref, rel * ref
        got = out[i:i + step].double()
        tol = (tol + half * want.abs() + tiny) * (1 + half)
        bad = ~((got - want).abs() <= tol)
        assert not bad.any(), (i, bad.nonzero()[:5].tolist())
    few = torch.empty((16, n), dtype=dtype, device="cuda")
    for i in sorted({0, m // 2, m - 16}):
        part = sp.Rows8(a8.q[i:i + 16], a8.e[i:i + 16], cols)
        assert torch.equal(sp.spdp_product8(state.h, part, b8, few, log=log), out[i:i + 16]), i


# Documents a workgroup takes by its own rule (16 for each fragment), rounds of words of a
# wavefront, and blocks of columns: all columns at once in LDS up to 32 / fragments of them, and
# part by part beyond.  Outputs above 64 MB whose rows start at multiples of 64 bytes are streamed.
PRODUCTS = [
    # m, n, cols, type, log, ld
    (200, 14724, 300, "f32", True, 14724),     # 2 fragments, 3 blocks
    (9000, 2048, 129, "f32", False, 2048),     # streamed, 2 blocks
    (65, 4100, 2100, "f32", True, 4100),       # 2, 17 blocks: two parts
    (300, 50000, 129, "f32", True, 50000),     # 4, 2 rounds, 2 blocks
    (300, 100016, 500, "f32", True, 100016),   # 4, 4 rounds, 4 blocks, streamed
    (300, 100001, 500, "bf16", True, 100007),  # 4, odd pitch
    (300, 50000, 1100, "bf16", True, 50000),   # 4, 9 blocks: two parts in each of 2 rounds
    (400, 100016, 300, "bf16", True, 100032),  # 6, 4 rounds, 3 blocks, streamed
    (777, 20000, 640, "f32", False, 20001),    # 6, 2 rounds, 5 blocks: the LDS full
    (777, 20011, 700, "f32", True, 20011),     # 6, 2 rounds, 6 blocks: two parts
    (2000, 10000, 1000, "f32", True, 10000),   # 6, streamed, two parts
    (777, 14724, 64, "f32", False, 14724),     # 8, 1 round
    (500, 50000, 500, "bf16", True, 50000),    # 8, 2 rounds, 4 blocks: the LDS full
    (1000, 50000, 513, "bf16", True, 50016),   # 8, 4 rounds, 5 blocks: two parts, streamed
    (1500, 20001, 1000, "f32", False, 20001),  # 8, 2 rounds, 8 blocks: two parts
    (97, 100016, 1500, "f32", True, 100016),   # 8, 12 blocks: three parts
    (2000, 100000, 500, "bf16", True, 100000),  # 8, 13 rounds, 4 blocks, streamed
    (1000, 100000, 200, "f32", False, 100000),  # 8, 7 rounds, streamed
]


@pytest.mark.parametrize("m,n,cols,type,log,ld", PRODUCTS)
def test_products_of_large_batches(state, m, n, cols, type, log, ld):
    say(f"product {m} x {n} x {cols} {type} log={log}, rows {ld} apart")
    _all_products(state, m, n, cols, type, log, ld)


@pytest.mark.parametrize("m,n,cols,ld", [(1, 5000, 50, 5000), (16, 1000, 300, 1003),
                                         (50, 3000, 500, 3001), (777, 14724, 64, 14724),
                                         (1000, 40000, 64, 40000)])
def test_product_of_probabilities_in_fp16(state, m, n, cols, ld):
    """Rows that add up to 1 against values up to 1: sums that fp16 holds."""
    say(f"probabilities {m} x {n} x {cols} in fp16")
    rng = np.random.default_rng(m + n)
    theta = rng.dirichlet(np.full(cols, 0.1), size=m)
    phi = rng.random((n, cols)) ** 8
    sides = [sp.spdp_pack8(state.h, dev(x), sp.Rows8.empty(*x.shape)) for x in (theta, phi)]
    a, b = (ow.unpack8(p.q.view(torch.uint8).cpu().numpy(), p.e.cpu().numpy()) for p in sides)
    out, buf = framed(m, n, torch.float16, ld=ld)
    sp.spdp_product8(state.h, *sides, out)
    some = np.unique(np.r_[0:min(m, 40), max(0, m - 40):m])
    _check_product(out[dev(some)].double().cpu().numpy(), a[some], b, False, torch.float16)
    assert frame_kept(buf, out)


@pytest.mark.parametrize("n", [2, 66])
def test_every_scale(state, n):
    """Every positive value at every scale times powers of two that bring it into fp32's
    range: itself for scales of 2^-124 to 2^119, rounded to bf16 beyond."""
    say(f"product, every scale, {n} words")
    e, code = np.meshgrid(np.arange(255), np.arange(127), indexing="ij")
    e, code = e.ravel(), code.ravel()
    q = np.zeros((len(e), 128), np.uint8)
    q[:, 0] = code
    a8 = sp.Rows8(dev(q).view(torch.float8_e4m3fn), dev(e[:, None].astype(np.uint8)), 1)
    value = np.ldexp(ow.VALUES8[code], e - 127)  # (fp64)
    # 8 bits of fraction at a time, and the steps of 2^-133 below bf16's normal range
    step = np.ldexp(1.0, np.maximum(np.frexp(value)[1] - 8, -133))
    rounded = np.rint(value / step) * step
    rounded[rounded >= 2.0 ** 128] = np.inf
    exact = (e >= 3) & (e <= 246)
    assert np.array_equal(rounded[exact], value[exact])
    power = np.where(np.arange(n) % 2 == 0, 100, -100)
    qb = np.zeros((n, 128), np.uint8)
    qb[:, 0] = 0x38  # 1
    b8 = sp.Rows8(dev(qb).view(torch.float8_e4m3fn), dev((power + 127)[:, None].astype(np.uint8)), 1)
    got = sp.spdp_product8(state.h, a8, b8, torch.empty((len(e), n), device="cuda")).cpu().numpy()
    for j in range(n):
        want = rounded * 2.0 ** power[j]
        want[want >= 2.0 ** 128] = np.inf
        normal = (want == 0) | (want >= 2.0 ** -126)  # (what a sum below fp32's range is, is its own)
        bad = normal & (got[:, j].astype(np.float64) != want)
        assert not bad.any(), (j, [(e[i], code[i], got[i, j], want[i]) for i in np.flatnonzero(bad)[:5]])


@pytest.mark.parametrize("n", [2, 66])
def test_scale_that_is_none(state, n):
    say(f"product, scale byte 255, {n} words")
    q = np.zeros((127, 256), np.uint8)
    q[:, 0], q[:, 1], q[:, 130] = np.arange(127), 0x38, 0x38
    e = np.full((127, 2), 127, np.uint8)
    e[:60, 0] = 255
    qb = np.zeros((n, 256), np.uint8)
    qb[:, 130] = 0x38
    a8, b8 = (sp.Rows8(dev(q).view(torch.float8_e4m3fn), dev(e), 200),
              sp.Rows8(dev(qb).view(torch.float8_e4m3fn), dev(np.full((n, 2), 127, np.uint8)), 200))
    got = sp.spdp_product8(state.h, a8, b8, torch.empty((127, n), device="cuda"))
    assert torch.isnan(got[:60]).all() and (got[60:] == 1).all()


@pytest.mark.parametrize("V", [100, 5000, 9000, 30000, 700000])
@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_draw_from_few_words(state, V, type):
    """Rows of which a mask, or scores of -inf, leave a few words here and there: most sums of
    16, 64 and 8 192 words are 0."""
    say(f"draw: few words of {V} {type}")
    rng = np.random.default_rng(V)
    rows, n = 10, 200 if V <= 30000 else 24
    x = _scores(rng, rows, V, TYPES[type])
    keep = np.zeros((rows, V), bool)
    for i, many in enumerate([1, 2, 3, 4, 5, 8, 20, 50, 100, 300]):
        keep[i, rng.integers(0, V, many)] = True
    keep[1, [V // 2, V // 2 + 1]] = True  # (neighbours, and both ends)
    keep[2, [0, V - 1]] = True
    bits = np.zeros((rows, -(-V // 32) * 32), np.uint8)
    bits[:, :V] = keep
    r = sp.Rules(rows, V, mask=dev(np.packbits(bits, axis=1, bitorder="little").view("<i4").copy()),
                 mask_of=dev(np.arange(rows, dtype=np.int32)))
    u = rng.random((rows, n))
    xo = np.where(keep, x.float().cpu().numpy(), -np.inf).astype(np.float32)
    for scores, rules in ((x, r), (dev(xo, TYPES[type]), None)):
        for uniforms in (u, np.where(np.arange(n) % 3 == 1, 1.0, u)):
            word, logp = _outs(rows, n)
            sp.spdp_draw(state.h, scores, word, logp, work_for(rows, V), u=dev(uniforms), rules=rules)
            _check_draws(word.cpu().numpy(), logp.cpu().numpy(), xo, uniforms, 1.0)


@pytest.mark.parametrize("at", [-690.0, -705.0, -709.0, -720.0, -735.0])
def test_draw_among_the_least_weights(state, at):
    """Uniforms among weights near and below fp64's normal range, in a chunk of words that hold
    no others."""
    say(f"draw: words of weight exp({at})")
    V = 20000
    x = np.full((1, V), -np.inf, np.float32)
    words = [10, 4000, 4001, 8000]
    x[0, words], x[0, V - 1] = at, 0.0
    x[0, 8192 + 5] = 1.0
    w = np.exp(at - 1.0)  # (fp64; half a weight is far more than what it is off by)
    total = 1.0 + np.exp(-1.0)
    u = np.array([[0.5, 1.5, 2.5, 3.5, 4.5]]) * (w / total)
    word, logp = _outs(1, 5)
    sp.spdp_draw(state.h, dev(x), word, logp, work_for(1, V), u=dev(u))
    assert word[0].tolist() == words + [8192 + 5]
    want = np.array([at - 1.0] * 4 + [0.0]) - np.log(total)
    np.testing.assert_allclose(logp[0].cpu().numpy(), want, rtol=2.0 ** -23)


def _hard_rows(rng, rows, V):
    """Rows that make choosing hard: ties at every height, rising and falling ones, a few words
    left here and there, runs without any, lone peaks, wide ranges."""
    x = rng.normal(size=(rows, V)).astype(np.float32) * 3
    for i in range(rows):
        kind = i % 9
        if kind == 0:
            x[i] = np.round(x[i])
        elif kind == 1:
            x[i] = np.arange(V) / 64.0
        elif kind == 2:
            x[i] = -np.arange(V) / 64.0
        elif kind == 3:
            x[i] = np.where(rng.random(V) < rng.choice([1e-3, 1e-2, 0.1]), x[i], -np.inf)
        elif kind == 4:
            for _ in range(6):
                a = rng.integers(0, V)
                x[i, a:a + rng.integers(1, max(2, V // 4))] = -np.inf
        elif kind == 5:
            x[i] = 2.0
            x[i, rng.integers(0, V, 3)] = 1.0
        elif kind == 6:
            x[i] = -np.inf
            a = rng.integers(0, max(1, V - 300))
            x[i, a:a + 300] = -1.0
        elif kind == 7:
            x[i] *= 60
        else:
            x[i, : V // 2] = -50.0
            x[i, rng.integers(0, V, 5)] = 40.0
    return x


def _best(x, k):
    """As ow.top, for many words."""
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -x), axis=1)[:, :k]
    value = np.full((len(x), k), -np.inf, np.float32)
    word = np.full((len(x), k), -1, np.int32)
    value[:, :order.shape[1]] = np.take_along_axis(x, order, 1)
    word[:, :order.shape[1]] = np.where(value[:, :order.shape[1]] > -np.inf, order, -1)
    return word, value


@pytest.mark.parametrize("rows,V", [(1100, 9000), (300, 20000), (18, 50000), (1030, 4100)])
@pytest.mark.parametrize("k", [1, 10, 256])
def test_top_of_hard_rows(state, rows, V, k):
    """Parts of one and of several chunks, with and without rules."""
    say(f"top {k} of {rows} x {V}, hard rows")
    rng = np.random.default_rng(V + k)
    x = _hard_rows(rng, rows, V)
    some = np.unique(np.r_[0:min(rows, 45), rows - 18:rows])
    r = RuleSet(rng, rows, V)
    for rules, want in ((None, x[some]), (r, None)):
        word, value = _outs(rows, k)
        sp.spdp_top(state.h, dev(x), word, value, work_for(rows, V, k), rules=rules and rules.c)
        if want is None:
            o = {n: (np.asarray(t)[some] if n != "listed" else [t[i] for i in some])
                 for n, t in r.o.items()}
            want = ow.adjusted(x[some], **o)
        ww, wv = _best(want, k)
        np.testing.assert_array_equal(word[dev(some)].cpu().numpy(), ww)
        np.testing.assert_array_equal(value[dev(some)].cpu().numpy(), wv)


@pytest.mark.parametrize("rows,V,n", [(27, 5000, 70), (18, 9000, 70), (9, 100000, 20), (300, 6000, 500)])
def test_draw_of_hard_rows(state, rows, V, n):
    say(f"draw {n} of {rows} x {V}, hard rows")
    rng = np.random.default_rng(V + n)
    x = _hard_rows(rng, rows, V)
    u = rng.random((rows, n))
    some = np.unique(np.r_[0:min(rows, 9), rows - 9:rows])
    r = RuleSet(rng, rows, V)
    for rules, temperature in ((None, 1.0), (r, 0.5)):
        word, logp = _outs(rows, n)
        sp.spdp_draw(state.h, dev(x), word, logp, work_for(rows, V), u=dev(u), temperature=temperature,
                     rules=rules and rules.c)
        want = x[some]
        if rules:
            o = {m: (np.asarray(t)[some] if m != "listed" else [t[i] for i in some])
                 for m, t in r.o.items()}
            want = ow.adjusted(x[some], **o)
        _check_draws(word[dev(some)].cpu().numpy(), logp[dev(some)].cpu().numpy(), want, u[some],
                     temperature)


def test_pack_of_blocks_without_numbers(state):
    say("pack: blocks of NaN and infinities only")
    rng = np.random.default_rng(5)
    x = rng.normal(size=(6, 400))
    x[0, :128], x[1, 128:256], x[2, 384:], x[3], x[4, ::2] = np.nan, np.inf, -np.inf, np.nan, np.inf
    for t in ("f64", "f32"):
        out = sp.spdp_pack8(state.h, dev(x, TYPES[t]), sp.Rows8.empty(6, 400))
        q, e = ow.pack8(dev(x, TYPES[t]).double().cpu().numpy())
        np.testing.assert_array_equal(out.e.cpu().numpy(), e)
        np.testing.assert_array_equal(ow.value8(out.q.view(torch.uint8).cpu().numpy()), ow.value8(q))


@pytest.mark.parametrize("m,n", [(17, 300), (300, 20000), (777, 10000), (1000, 14724)])
def test_product_keeps_rows_apart(state, m, n):
    """NaN, zeros and negative values of one document or word are seen in its own scores only."""
    say(f"product {m} x {n}: rows apart")
    (a8, _), (b8, _) = _model8(state, 3, m, n, 300)
    out = sp.spdp_product8(state.h, a8, b8, torch.empty((m, n), device="cuda"), log=True)
    assert torch.isfinite(out).all()
    docs, words = [0, m // 2, m - 1], [0, 63, 64, n // 2, n - 65, n - 1]
    a, b = a8.q.view(torch.uint8), b8.q.view(torch.uint8)
    a[docs[0], 299] = 127
    a[docs[1]] = 0
    a[docs[2]] |= 128
    b[words[0], 0] = 255
    b[words[1]] = 0
    b[words[2]] |= 128
    b[words[3], 150] = 127
    b[words[4]] |= 128
    b[words[5]] = 0
    got = sp.spdp_product8(state.h, a8, b8, torch.empty((m, n), device="cuda"), log=True)
    keep_d, keep_w = torch.ones(m, dtype=torch.bool), torch.ones(n, dtype=torch.bool)
    keep_d[docs], keep_w[words] = False, False
    assert torch.equal(got[keep_d.cuda()][:, keep_w.cuda()], out[keep_d.cuda()][:, keep_w.cuda()])
    w = keep_w.cuda()
    assert torch.isnan(got[docs[0]]).all()
    assert torch.isneginf(got[docs[1]][w]).all() and torch.isnan(got[docs[2]][w]).all()
    d = keep_d.cuda()
    nan, zero = [words[i] for i in (0, 2, 3, 4)], [words[i] for i in (1, 5)]
    assert torch.isnan(got[d][:, nan]).all() and torch.isneginf(got[d][:, zero]).all()
    # negative documents and words make positive sums
    assert torch.equal(got[docs[2]][[words[2], words[4]]], out[docs[2]][[words[2], words[4]]])


@pytest.mark.parametrize("V,step,temperature", [(20000, 1 / 64, 0.05), (20000, -1 / 64, 0.05),
                                                (30000, 1 / 256, 0.01), (9000, -0.5, 1.0),
                                                (9000, 0.5, 1.0), (700000, 2.0 ** -13, 2.0 ** -6)])
def test_draw_ends_of_slopes(state, V, step, temperature):
    """Rows that rise or fall: around the first and the last word with weight stand many that
    have some together and none each."""
    say(f"draw: ends of a slope of {step} over {V} words at {temperature}")
    x = np.stack([np.arange(V) * step, np.arange(V) * step + 0.3 * np.sin(np.arange(V))]).astype(np.float32)
    u = np.tile(np.array([0.0, 1.0, 0.5] * 30 + [-1.0, 2.0]), (2, 1))
    rng = np.random.default_rng(V)
    words = rng.integers(0, V, 4000)
    r = sp.Rules(2, V, doc_off=dev(np.array([0, 1000, 4000])), words=dev(words.astype(np.int32)),
                 penalties=dev(np.tile(np.array([1.0, 0.5 * abs(step), 0.0], np.float32), (2, 1))))
    for rules in (None, r):
        xo = x if rules is None else ow.adjusted(x, [words[:1000], words[1000:]],
                                                 [[1.0, 0.5 * abs(step), 0.0]] * 2)
        word, logp = _outs(2, 92)
        sp.spdp_draw(state.h, dev(x), word, logp, work_for(2, V), u=dev(u), rules=rules,
                     temperature=temperature)
        with np.errstate(under="ignore"):
            z = (xo.astype(np.float64) - xo.max(1, keepdims=True).astype(np.float64)) / temperature
            law = np.exp(z)
        for i in range(2):
            # (words whose weight lies at the border of what fp64 rounds to 0 are as good as those
            # next to them: the logarithm of 2^-1075 to 1e-9)
            sure, any_ = z[i] > -1075 * np.log(2) + 1e-9, z[i] > -1075 * np.log(2) - 1e-9
            got = word[i].cpu().numpy()
            for t, of in ((0, 0), (1, -1)):
                ends = {int(np.flatnonzero(m)[of]) for m in (sure, any_)}
                assert set(got[t:90:3].tolist()) | {int(got[90 + t])} <= ends, (i, t, ends, got[t])
            c = np.cumsum(law[i].astype(np.longdouble))
            assert (got[2:90:3] == np.searchsorted(c, 0.5 * c[-1], side="right")).all()
