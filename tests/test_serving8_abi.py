"""Refusals of the calls over caches of 8 bits and of the logits' adjustment,
checked on the host before any HIP call: no GPU is needed, and the pointers used
here are never dereferenced.  And the CPU oracle of these operations against
exact arithmetic and closed forms."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import serving as OS
from paper_2605_08755_amd import laq
from test_serving_abi import FAKE, FIELDS, GOOD, KMAX, KMIN, Batch

GOOD8 = dict(GOOD, page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128)


@pytest.fixture(scope="module")
def L():
    return laq.lib()


def batch(**kw):
    v = dict(GOOD8, **kw)
    return ctypes.byref(Batch(*[v[n] for n in FIELDS]))


def append(L, b=None, ks=FAKE, vs=FAKE, qkv=FAKE, stride=48 * 128, qw=FAKE, kw=FAKE, cs=FAKE, rope=100, Hq=32, Hkv=8,
           d=128, eps=1e-6, q_out=FAKE, **kw_b):
    return L.laq_paged_append_e4m3(batch(**kw_b) if b is None else b, ks, vs, qkv, stride, qw, kw, cs, rope, Hq, Hkv, d,
                                   eps, q_out, None)


def attention(L, b=None, ks=FAKE, vs=FAKE, q=FAKE, Hq=32, Hkv=8, d=128, window=0, out=FAKE, ws=FAKE, nbytes=1 << 30,
              **kw_b):
    return L.laq_paged_attention_e4m3(batch(**kw_b) if b is None else b, ks, vs, q, Hq, Hkv, d, window, out, ws, nbytes,
                                      None)


@pytest.mark.parametrize("call", [append, attention])
def test_batch_refusals(L, call):
    name = b"laq_paged_append_e4m3" if call is append else b"laq_paged_attention_e4m3"
    assert call(L, b=ctypes.c_void_p(0)) == laq.LAQ_ERR_NULL_POINTER
    for f in FIELDS[:5]:
        assert call(L, **{f: 0}) == laq.LAQ_ERR_NULL_POINTER
        assert name in L.laq_last_error()
    for f in ("ks", "vs"):
        assert call(L, **{f: 0}) == laq.LAQ_ERR_NULL_POINTER
        assert name in L.laq_last_error()
    for f, values in (("num_pages", (0, -1, KMIN, 1 << 31, KMAX)),
                      ("page_size", (0, -16, 1, 8, 15, 24, 17, 1 << 21, KMAX, KMIN)),
                      ("page_stride", (0, -128, 64, KMAX, KMIN)), ("head_stride", (0, -8, 120, KMAX)),
                      ("slot_stride", (0, 64, -128, (1 << 26) + 16, KMAX, KMIN)),
                      ("table_pages", (0, -1, 1 << 27, KMAX, KMIN)), ("table_stride", (3, -1, KMIN, KMAX)),
                      ("B", (-1, (1 << 20) + 1, KMAX, KMIN)), ("T", (-1, (1 << 30) + 1, 1 << 26, KMAX, KMIN))):
        for v in values:
            assert call(L, **{f: v}) == laq.LAQ_ERR_BAD_SHAPE, (f, v)
    for f in ("page_stride", "head_stride", "slot_stride"):  # rows of codes start at 16 bytes
        assert call(L, **{f: GOOD8[f] + 8}) == laq.LAQ_ERR_MISALIGNED
    for f, o in (("k_pages", 8), ("v_pages", 2), ("page_table", 2), ("token_start", 1), ("seq_len", 2)):
        assert call(L, **{f: FAKE + o}) == laq.LAQ_ERR_MISALIGNED
    for Hq, Hkv in ((0, 1), (8, 0), (8, 3), (-8, -8), (4104, 8), (KMAX, 1), (8, KMIN), (KMIN, 1)):
        assert call(L, Hq=Hq, Hkv=Hkv) == laq.LAQ_ERR_BAD_SHAPE
    for d in (64, 0, 127, KMAX):
        assert call(L, d=d) == laq.LAQ_ERR_BAD_SHAPE
    nothing = {f: 0 for f in FIELDS[:5]}
    assert call(L, B=0, ks=0, vs=0, **nothing) == laq.LAQ_OK and call(L, T=0, ks=0, vs=0, **nothing) == laq.LAQ_OK
    assert call(L, T=0, page_size=8, **nothing) == laq.LAQ_ERR_BAD_SHAPE


def test_append_refusals(L):
    for f in ("qkv", "cs", "q_out"):
        assert append(L, **{f: 0}) == laq.LAQ_ERR_NULL_POINTER
    for v in (0, -1, KMIN, (1 << 31) + 1, KMAX):
        assert append(L, rope=v) == laq.LAQ_ERR_BAD_SHAPE
    for v in (48 * 128 - 8, 0, -48 * 128, KMAX, KMIN):
        assert append(L, stride=v) == laq.LAQ_ERR_BAD_SHAPE
    assert append(L, stride=48 * 128 + 4) == laq.LAQ_ERR_MISALIGNED
    for v in (-1e-6, math.inf, math.nan):
        assert append(L, eps=v) == laq.LAQ_ERR_BAD_SHAPE
    for f, o in (("qkv", 8), ("qw", 2), ("kw", 8), ("cs", 2), ("q_out", 4)):
        assert append(L, **{f: FAKE + o}) == laq.LAQ_ERR_MISALIGNED
    # windows of 16 rows: 2 x 4096 + 1 waves of 64 threads each
    assert append(L, Hq=4096, Hkv=4096, stride=3 * 4096 * 128, T=1 << 18) == laq.LAQ_ERR_BAD_SHAPE
    assert b"too many rows" in L.laq_last_error()


def test_attention_refusals(L):
    big = dict(table_pages=1000, table_stride=1000)
    need = L.laq_paged_attention_e4m3_workspace_bytes(2, 3, 32, 8, 16000)
    assert need > 0
    for f in ("q", "out"):
        assert attention(L, **{f: 0}) == laq.LAQ_ERR_NULL_POINTER
    assert attention(L, ws=0, **big) == laq.LAQ_ERR_NULL_POINTER
    for v in (need - 1, 0, -1, KMIN):
        assert attention(L, nbytes=v, **big) == laq.LAQ_ERR_BAD_SHAPE
    for v in (-1, KMIN, (1 << 30) + 1, KMAX):
        assert attention(L, window=v) == laq.LAQ_ERR_BAD_SHAPE
    for f, o in (("q", 8), ("out", 2), ("ws", 8)):
        assert attention(L, **{f: FAKE + o}) == laq.LAQ_ERR_MISALIGNED
    for Hq, Hkv, B, T in ((1024, 1024, 1 << 20, 1 << 20), (16, 16, 1 << 20, (1 << 26) - 1)):
        assert attention(L, Hq=Hq, Hkv=Hkv, B=B, T=T) == laq.LAQ_ERR_BAD_SHAPE


def test_attention_workspace_query(L):
    f, f16 = L.laq_paged_attention_e4m3_workspace_bytes, L.laq_paged_attention_workspace_bytes
    for args in ((0, 1, 8, 8, 100), (1, 0, 8, 8, 100), (1, 1, 0, 8, 100), (1, 1, 8, 3, 100), (1, 1, 8, 8, 0),
                 (KMAX, 1, 8, 8, 100), (1, KMAX, 8, 8, 100), (1, 1, KMAX, 1, 100), (1, 1, 8, KMIN, 100),
                 (1, 1, 8, 8, KMAX), (KMIN, KMIN, KMIN, KMIN, KMIN)):
        assert f(*args) == 0
    assert f(1, 1, 64, 8, 512) == 0 < f(1, 1, 64, 8, 1024)  # not split; split
    for Hkv in (1, 2, 3, 8, 40, 512, 4096):
        for R in (1, 3, 5, 8, 24):
            for B in (1, 2, 3, 7, 64, 65, 300):
                for T in (1, 2, 16, 17, 33, 129, 700, 5000, 40000):
                    for capacity in (16, 300, 600, 1100, 4096, 1 << 20, 1 << 30):
                        if Hkv * R <= 4096:
                            assert 0 <= f(B, T, Hkv * R, Hkv, capacity) <= f16(B, T, Hkv * R, Hkv, capacity), (B, T, R, Hkv)


ADJUST = ("history", "history_len", "prompt_len", "history_stride", "history_room", "repetition", "frequency", "presence",
          "bias_token", "bias_value", "bias_stride", "biases", "mask", "mask_stride")
NUMBERS = ("history_stride", "history_room", "bias_stride", "biases", "mask_stride")
GOOD_ADJUST = dict({n: FAKE for n in ADJUST}, history_stride=100, history_room=100, bias_stride=5, biases=5, mask_stride=32)


class Adjust(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64 if n in NUMBERS else ctypes.c_void_p) for n in ADJUST]


def adjust(L, a=None, logits=FAKE, stride=1000, rows=4, V=1000, out=2 * FAKE, out_stride=1000, **kw):
    v = dict(GOOD_ADJUST, **kw)
    s = ctypes.byref(Adjust(*[v[n] for n in ADJUST])) if a is None else a
    return L.laq_adjust_logits_f16(s, logits, stride, rows, V, out, out_stride, None)


def test_adjust_refusals(L):
    assert laq._LOGITS_ADJUST.size == ctypes.sizeof(Adjust) == 14 * 8
    assert adjust(L, a=ctypes.c_void_p(0)) == laq.LAQ_ERR_NULL_POINTER
    for kw in (dict(logits=0), dict(out=0), dict(history_len=0), dict(bias_value=0)):
        assert adjust(L, **kw) == laq.LAQ_ERR_NULL_POINTER
        assert b"laq_adjust_logits_f16" in L.laq_last_error()
    for f, values in (("V", (0, -1, (1 << 24) + 1, KMAX, KMIN)), ("rows", (-1, 1 << 22, KMAX, KMIN)),
                      ("stride", (999, 0, -1000, (1 << 32) + 1, KMAX, KMIN)),
                      ("out_stride", (999, 0, -1000, (1 << 32) + 1, KMAX, KMIN)),
                      ("history_room", (-1, 1 << 20, KMAX, KMIN)), ("history_stride", (-1, (1 << 32) + 1, KMAX, KMIN)),
                      ("biases", (-1, laq.MAX_BIASES + 1, KMAX, KMIN)), ("bias_stride", (-1, (1 << 32) + 1, KMAX, KMIN)),
                      ("mask_stride", (-1, (1 << 32) + 1, KMAX, KMIN))):
        for v in values:
            assert adjust(L, **{f: v}) == laq.LAQ_ERR_BAD_SHAPE, (f, v)
    for f in ("logits", "out"):
        assert adjust(L, **{f: 3 * FAKE + 1}) == laq.LAQ_ERR_MISALIGNED
    for f in set(ADJUST) - set(NUMBERS):
        assert adjust(L, **{f: FAKE + 2}) == laq.LAQ_ERR_MISALIGNED
    # out over a part of the logits, or over all of them with other strides
    for kw in (dict(out=FAKE + 2), dict(out=FAKE - 2), dict(out=FAKE + 2 * 4 * 1000 - 2), dict(out=FAKE, out_stride=1001),
               dict(out=FAKE, rows=1, stride=0, out_stride=0, V=1 << 24, logits=FAKE + 16)):
        assert adjust(L, **kw) == laq.LAQ_ERR_BAD_SHAPE, kw
    # 2^22 - 1 rows of 2^24 logits
    assert adjust(L, rows=(1 << 22) - 1, V=1 << 24, stride=1 << 24, out_stride=1 << 24, out=1 << 60) == laq.LAQ_ERR_BAD_SHAPE
    assert b"too many" in L.laq_last_error()
    assert adjust(L, rows=0, logits=0, out=0) == laq.LAQ_OK


# ---------------------------------------------------------------------------
# the oracle
# ---------------------------------------------------------------------------
def test_oracle_codes():
    """Against exact rational arithmetic: the nearest code, of two the even one."""
    v = OS.e4m3_values()
    assert v[0x38] == 1 and v[0x7E] == 448 and v[1] == 2.0**-9 and np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and v[0xB8] == -1
    rng = np.random.default_rng(0)
    mids = [(v[c] + v[c + 1]) / 2 for c in range(126)]
    xs = list(v[:127]) + mids + [m * (1 + s * 2.0**-40) for m in mids for s in (-1, 1)] + list(rng.standard_normal(300) * 100)
    exact = [Fraction(float(x)) for x in v[:127]]
    for x in xs:
        got = int(OS.e4m3(x))
        a = Fraction(abs(float(x)))
        far = [abs(e - a) for e in exact]
        best = min(far)
        want = [c for c in range(127) if far[c] == best]
        assert (got & 127) == (want[0] if len(want) == 1 else [c for c in want if c % 2 == 0][0]), x
        assert (got >> 7) == (math.copysign(1, x) < 0)
    assert [int(OS.e4m3(x)) for x in (500.0, -1e30, math.inf, math.nan)] == [0x7E, 0xFE, 0x7F, 0x7F]


def test_oracle_scales():
    for a, s in ((0.0, 112), (448 * 2.0**-15, 112), (448.0001 * 2.0**-15, 113), (448.0, 127), (448.1, 128), (57344.0, 134),
                 (1e9, 134), (1.75, 119), (1.76, 120)):
        assert OS.least_scale(a) == s


def test_oracle_append():
    """One row into a block that holds another: the scale grows to hold it and
    the other's codes are rounded again; into a fresh block the old scale is
    forgotten; the values are those of the fp16 append, rounded."""
    rng = np.random.default_rng(3)
    Hq, Hkv, ps = 2, 1, 16
    cs = np.concatenate([np.ones((40, 64)), np.zeros((40, 64))], axis=1)
    qkv = rng.standard_normal((1, 512))
    qkv[0, 300] = 30.0
    codes = np.full((2, Hkv, ps, 128), 0x35, dtype=np.uint8)  # 0.8125
    scales = np.full((2, Hkv, 1), 119, dtype=np.uint8)
    empty = np.zeros((1, Hq, 128))
    q, ((kc, ks, _), (vc, vs, _)) = OS.paged_append_e4m3(qkv, None, None, cs, ((codes, scales), (codes, scales)),
                                                         np.array([[1, 0]]), [0, 1], [4], Hq, 1e-6, empty)
    assert 1.75 < np.abs(qkv[0, 384:]).max() <= 3.5
    assert ks[1, 0, 0] == 124 and vs[1, 0, 0] == 120 and ks[0, 0, 0] == 119  # 28 < 30 <= 56
    assert (kc[1, 0, :3] == OS.e4m3(0.8125 / 32)).all() and (vc[1, 0, :3] == 0x2D).all() and (kc[1, 0, 4:] == 0x35).all()
    k = OS.cache_values(kc, ks)[1, 0, 3]
    assert np.abs(k - qkv[0, 256:384]).max() <= 1.0 and k[44] == 30.0
    assert np.allclose(q[0], qkv[0, :256].reshape(2, 128))
    _, ((kc, ks, _), _) = OS.paged_append_e4m3(qkv / 1000, None, None, cs, ((codes, scales), (codes, scales)),
                                               np.array([[1, 0]]), [0, 1], [17], Hq, 1e-6, empty)
    assert ks[0, 0, 0] == 114 and (kc[0, 0, 1:] == 0x35).all() and (kc[1] == 0x35).all()


def test_oracle_adjust():
    x = [2.0, -2.0, 1.0, 0.0, 5.0]
    got = OS.adjust_row(x, [0, 1, 1, 2, 9, -1], 1, 2.0, 0.5, 0.25, [(4, 1.0), (4, -3.0), (3, 0.5)], None)
    assert got.tolist() == [1.0, -4.0 - 1.0 - 0.25, 0.5 - 0.5 - 0.25, 0.5, 2.0]
    assert OS.adjust_row(x, mask=[0b10011]).tolist() == [2.0, -2.0, -math.inf, -math.inf, 5.0]
