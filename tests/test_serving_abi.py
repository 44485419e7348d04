"""Refusals of the batched serving entry points (paged append, paged
attention, sampling), checked on the host before any HIP call: no GPU is
needed, and the pointers used here are never dereferenced.  And the CPU
oracle of these operations against closed forms."""
import ctypes
import math

import numpy as np
import pytest

from oracle import decode as OD
from oracle import serving as OS
from paper_2605_08755_amd import laq

FAKE = 0x100000  # 16-byte aligned, never dereferenced
KMAX, KMIN = 2**63 - 1, -2**63

FIELDS = ("k_pages", "v_pages", "page_table", "token_start", "seq_len", "num_pages", "page_size", "page_stride",
          "head_stride", "slot_stride", "table_pages", "table_stride", "B", "T")
GOOD = dict(k_pages=FAKE, v_pages=FAKE, page_table=FAKE, token_start=FAKE, seq_len=FAKE, num_pages=10, page_size=16,
            page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128, table_pages=4, table_stride=4, B=2, T=3)


class Batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p if i < 5 else ctypes.c_int64) for i, n in enumerate(FIELDS)]


@pytest.fixture(scope="module")
def L():
    return laq.lib()


def batch(**kw):
    v = dict(GOOD, **kw)
    return ctypes.byref(Batch(*[v[n] for n in FIELDS]))


def append(L, b=None, qkv=FAKE, stride=48 * 128, qw=FAKE, kw=FAKE, cs=FAKE, rope=100, Hq=32, Hkv=8, d=128, eps=1e-6,
           q_out=FAKE, **kw_b):
    return L.laq_paged_append_f16(batch(**kw_b) if b is None else b, qkv, stride, qw, kw, cs, rope, Hq, Hkv, d, eps,
                                  q_out, None)


def attention(L, b=None, q=FAKE, Hq=32, Hkv=8, d=128, window=0, out=FAKE, ws=FAKE, nbytes=1 << 30, **kw_b):
    return L.laq_paged_attention_f16(batch(**kw_b) if b is None else b, q, Hq, Hkv, d, window, out, ws, nbytes, None)


def sample(L, logits=FAKE, stride=1000, rows=4, V=1000, u=FAKE, t=FAKE, k=FAKE, p=FAKE, m=FAKE, token=FAKE, prob=FAKE):
    return L.laq_sample_f16(logits, stride, rows, V, u, t, k, p, m, token, prob, None)


def test_struct_matches_the_header():
    assert laq._PAGED_BATCH.size == ctypes.sizeof(Batch) == 14 * 8


@pytest.mark.parametrize("call", [append, attention])
def test_batch_refusals(L, call):
    name = b"laq_paged_append_f16" if call is append else b"laq_paged_attention_f16"
    assert call(L, b=ctypes.c_void_p(0)) == laq.LAQ_ERR_NULL_POINTER
    for f in FIELDS[:5]:
        assert call(L, **{f: 0}) == laq.LAQ_ERR_NULL_POINTER
        assert name in L.laq_last_error()
    for f, values in (("num_pages", (0, -1, KMIN, 1 << 31, KMAX)),
                      ("page_size", (0, -16, 1, 8, 15, 24, 17, 1 << 21, KMAX, KMIN)),
                      ("page_stride", (0, -128, 64, KMAX, KMIN)), ("head_stride", (0, -8, 120, KMAX)),
                      ("slot_stride", (0, 64, -128, (1 << 26) + 8, KMAX, KMIN)),
                      ("table_pages", (0, -1, 1 << 27, KMAX, KMIN)), ("table_stride", (3, -1, KMIN, KMAX)),
                      ("B", (-1, (1 << 20) + 1, KMAX, KMIN)), ("T", (-1, (1 << 30) + 1, 1 << 26, KMAX, KMIN))):
        for v in values:
            assert call(L, **{f: v}) == laq.LAQ_ERR_BAD_SHAPE, (f, v)
    for f in ("page_stride", "head_stride", "slot_stride"):
        assert call(L, **{f: GOOD[f] + 4}) == laq.LAQ_ERR_MISALIGNED
    for f, o in (("k_pages", 8), ("v_pages", 2), ("page_table", 2), ("token_start", 1), ("seq_len", 2)):
        assert call(L, **{f: FAKE + o}) == laq.LAQ_ERR_MISALIGNED
    for Hq, Hkv in ((0, 1), (8, 0), (8, 3), (-8, -8), (4104, 8), (KMAX, 1), (8, KMIN), (KMIN, 1)):
        assert call(L, Hq=Hq, Hkv=Hkv) == laq.LAQ_ERR_BAD_SHAPE
    for d in (64, 0, 127, KMAX):
        assert call(L, d=d) == laq.LAQ_ERR_BAD_SHAPE
    # an empty batch: done, whatever its pointers are; its sizes are checked all the same
    nothing = {f: 0 for f in FIELDS[:5]}
    assert call(L, B=0, **nothing) == laq.LAQ_OK and call(L, T=0, **nothing) == laq.LAQ_OK
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


def test_attention_refusals(L):
    # enough pages for a sequence's positions to be split: a workspace is needed
    big = dict(table_pages=1000, table_stride=1000)
    need = L.laq_paged_attention_workspace_bytes(2, 3, 32, 8, 16000)
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


def test_launch_size_refusals(L):
    """What would take 2^32 threads or more is refused, not left to the launch."""
    for call in (append, attention):
        assert call(L, Hq=1, Hkv=1, T=1 << 26) == laq.LAQ_ERR_BAD_SHAPE
    for Hq, Hkv, B, T in ((1024, 1024, 1 << 20, 1 << 20), (16, 16, 1 << 20, (1 << 26) - 1)):
        assert attention(L, Hq=Hq, Hkv=Hkv, B=B, T=T) == laq.LAQ_ERR_BAD_SHAPE
        assert b"too many rows" in L.laq_last_error()
    assert sample(L, rows=1 << 22) == laq.LAQ_ERR_BAD_SHAPE


def test_attention_workspace_query(L):
    f = L.laq_paged_attention_workspace_bytes
    for args in ((0, 1, 8, 8, 100), (1, 0, 8, 8, 100), (1, 1, 0, 8, 100), (1, 1, 8, 3, 100), (1, 1, 8, 8, 0),
                 (KMAX, 1, 8, 8, 100), (1, KMAX, 8, 8, 100), (1, 1, KMAX, 1, 100), (1, 1, 8, KMIN, 100),
                 (1, 1, 8, 8, KMAX), (KMIN, KMIN, KMIN, KMIN, KMIN)):
        assert f(*args) == 0
    assert f(4, 4, 32, 8, 128) == 0  # a single range: nothing to join
    for B, T, Hq, Hkv in ((1, 1, 32, 8), (64, 64, 64, 8), (3, 5000, 40, 8), (1, 1 << 18, 32, 8), (7, 9, 4096, 4096),
                          (1000, 1000, 1, 1), (1, 3, 4096, 1)):
        last = 0
        for capacity in (16, 4096, 1 << 20, 1 << 30):  # a longer table never needs less, and it stays bounded
            n = f(B, T, Hq, Hkv, capacity)
            assert last <= n <= 140 * 10**6, (B, T, Hq, Hkv, capacity, n)
            last = n


def test_sample_refusals(L):
    for f in ("logits", "u", "token"):
        assert sample(L, **{f: 0}) == laq.LAQ_ERR_NULL_POINTER
        assert b"laq_sample_f16" in L.laq_last_error()
    for v in (0, -1, (1 << 24) + 1, KMAX, KMIN):
        assert sample(L, V=v) == laq.LAQ_ERR_BAD_SHAPE
    for v in (-1, 1 << 31, KMAX, KMIN):
        assert sample(L, rows=v) == laq.LAQ_ERR_BAD_SHAPE
    for v in (999, 0, -1000, (1 << 32) + 1, KMAX, KMIN):
        assert sample(L, stride=v) == laq.LAQ_ERR_BAD_SHAPE
    assert sample(L, logits=FAKE + 1) == laq.LAQ_ERR_MISALIGNED
    for f in ("u", "t", "k", "p", "m", "token", "prob"):
        assert sample(L, **{f: FAKE + 2}) == laq.LAQ_ERR_MISALIGNED
    assert sample(L, rows=0, logits=0, u=0, token=0) == laq.LAQ_OK


# ---------------------------------------------------------------------------
# the oracle
# ---------------------------------------------------------------------------
def test_oracle_attention_is_the_single_token_one():
    """One sequence in order of its pages: oracle/decode.py's attention; the
    rows of a chunk see what each would see alone; a window drops the rest."""
    rng = np.random.default_rng(1)
    Hq, Hkv, L, ps = 4, 2, 37, 16
    K, V = rng.standard_normal((2, Hkv, L, 128))
    q = rng.standard_normal((3, Hq, 128))
    table = np.array([[2, 0, 1]])
    kp, vp = np.full((2, 3, Hkv, ps, 128), np.nan)
    for t in range(L):
        kp[table[0, t // ps], :, t % ps], vp[table[0, t // ps], :, t % ps] = K[:, t], V[:, t]
    out, _, _ = OS.paged_attention(q, kp, vp, table, [0, 3], [L], 0, np.zeros((3, Hq, 128)))
    win, _, _ = OS.paged_attention(q, kp, vp, table, [0, 3], [L], 5, np.zeros((3, Hq, 128)))
    for i in range(3):
        n = L - 2 + i
        assert np.allclose(out[i], OD.decode_attention(q[i], K[:, :n], V[:, :n]), rtol=1e-12, atol=1e-12)
        assert np.allclose(win[i], OD.decode_attention(q[i], K[:, n - 5:n], V[:, n - 5:n]), rtol=1e-12, atol=1e-12)


def test_oracle_append_is_the_single_token_one():
    rng = np.random.default_rng(2)
    Hq, Hkv, pos = 4, 2, 21
    qkv = rng.standard_normal((1, (Hq + 2 * Hkv) * 128))
    qw, kw = rng.standard_normal((2, 128))
    a = np.array([OD.rope_angles(p, 128, 1e6) for p in range(40)])
    cs = np.concatenate([np.cos(a), np.sin(a)], axis=1)
    z = np.zeros((4, Hkv, 16, 128))
    q, k, v = OS.paged_append(qkv, qw, kw, cs, z, z, np.array([[3, 1]]), [0, 1], [pos + 1], Hq, 1e-6,
                              np.zeros((1, Hq, 128)))
    rq, rk, rv = OD.qk_norm_rope(qkv, qw, kw, pos, Hq, Hkv, 128, 1e-6, 1e6)
    assert np.allclose(q[0], rq, rtol=1e-12) and np.allclose(k[1, :, 5], rk, rtol=1e-12)
    assert np.array_equal(v[1, :, 5], rv) and np.count_nonzero(k.any(axis=(1, 3))) == 1


def test_oracle_sample_by_hand():
    """Weights 4 : 2 : 2 : 1 (equal logits in index order), T = 1."""
    x = np.log([2.0, 4.0, 1.0, 2.0])
    walk = lambda **kw: [OS.sample_row(x, u, **kw)[0] for u in (0, 0.43, 0.45, 0.66, 0.67, 0.88, 0.9, 1.0)]  # noqa: E731
    assert walk() == [1, 1, 0, 0, 3, 3, 2, 2]
    assert walk(top_k=2) == [1, 1, 1, 1, 0, 0, 0, 0]            # 4 : 2
    assert walk(top_p=0.5) == [1, 1, 1, 1, 0, 0, 0, 0]          # 4 of 9 is less, 6 of 9 is not
    assert walk(top_p=0.4) == [1] * 8
    assert walk(min_p=0.3) == [1, 1, 1, 0, 0, 3, 3, 3]          # 4 : 2 : 2
    assert walk(temperature=0.0, top_k=3) == [1] * 8
    assert OS.sample_row(x, 0.5)[1] == pytest.approx(2 / 9)
    assert OS.sample_row([-np.inf, np.nan], 0.5) == (-1, 0.0)
    assert OS.sample_row([-np.inf, 3.0, np.nan], 0.99, top_k=3) == (1, 1.0)
