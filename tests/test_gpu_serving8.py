"""Batched serving over caches of 8 bits on the GPU (append, attention), and
logits before sampling, against the float64 oracle (oracle/serving.py).

Tolerances, from the arithmetic:
  append     q as paged_append's: fp32 steps on fp16 inputs, one fp16 rounding
             (linear_check).  Values are fp16 numbers, so their codes are the oracle's, and so are scales and the codes of
             earlier positions.  A key before rounding is off by the norm (a sum
             of 128 squares in fp32, 128 x 2^-24 of it, half of that in the root;
             a few more roundings) and the rotation, each relative to the pair's
             magnitude: 2^-16 of it covers both.  Its code is one nearest to a
             value within that: half a step of the code, plus that.
  attention  what the cache stands for are fp16 numbers, so the tolerance is that
             of the attention over an fp16 cache (tests/test_gpu_serving.py), and
             2^-20 of the weights where probabilities are two fp16 numbers (11
             bits each, the first cut off, the second too).
  adjust     fp32 steps: the reciprocal of the repetition and the product with
             it, frequency times count, two differences, the bias: six, each off
             by 2^-24 of its result, and one rounding to fp16 (2^-11).
"""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from oracle.compare import linear_check
from paper_2605_08755_amd import decode, laq
from test_gpu_serving import SHAPE, Batch, attention_check, dev, f16, make_step, say, set_rows

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
EPS = 1e-6
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def codes_dev(c, slot_major=False):
    if slot_major:
        return dev(c.transpose(0, 2, 1, 3)).transpose(1, 2).view(E4M3)
    return dev(c).view(E4M3)


def host(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


class Batch8(Batch):
    """A batch whose caches are codes (kc, vc) with scales (ks, vs), magnitudes
    of every block its own; k and v are the fp16 values that they stand for."""

    def __init__(self, rng, tokens, before, ps, Hkv, garbage=0x7F, spread=2, **kw):
        super().__init__(rng, tokens, before, ps, Hkv, garbage=None, **kw)
        shape = (self.P, Hkv, ps // 16)
        self.ks, self.vs = (rng.integers(118 - spread, 119 + spread, shape).astype(np.uint8) for _ in range(2))
        self.kc, self.vc = (OS.e4m3(rng.standard_normal((self.P, Hkv, ps, 128)) * 150) for _ in range(2))
        if garbage is not None:
            for c in (self.kc, self.vc):
                c[np.broadcast_to(~self.used[:, None], (self.P, Hkv, ps))] = garbage
        self.values()

    def values(self):
        with np.errstate(invalid="ignore"):
            self.k, self.v = (OS.cache_values(c, s).astype(np.float16) for c, s in ((self.kc, self.ks), (self.vc, self.vs)))

    def device8(self):
        return (codes_dev(self.kc, self.slot_major), codes_dev(self.vc, self.slot_major), dev(self.ks).view(E8M0),
                dev(self.vs).view(E8M0), dev(self.table), dev(self.start), dev(self.lens))


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
def half_step(x):
    """Half the distance of the codes around |x| (in the codes' units)."""
    return np.ldexp(0.5, np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0**-20))), -6).astype(int) - 3)


def check_append(rng, bt, qkv, qw, kw, cs, Hq, q_canary, got=None):
    """Runs the append on the batch's caches and compares all that it writes; returns the caches after it."""
    if got is None:
        k, v, ks, vs, table, start, lens = bt.device8()
        q = dev(q_canary)
        args = (None if qw is None else dev(qw), None if kw is None else dev(kw), cs)
        out = laq.paged_append_e4m3(dev(qkv), *args, k, v, ks, vs, table, start, lens, Hq, EPS, q_out=q)
        assert out is q
        torch.cuda.synchronize()
        q_host = q.cpu().numpy()
        got = (host(k), host(ks)), (host(v), host(vs))
    else:
        q_host = None
    q_want, want = OS.paged_append_e4m3(qkv, qw, kw, cs.cpu().numpy(), ((bt.kc, bt.ks), (bt.vc, bt.vs)), bt.table, bt.start,
                                   bt.lens, Hq, EPS, q_canary)
    if q_host is not None:
        r = linear_check(q_host, q_want)
        assert r["ok"], r
        rows = [r for r, _, _ in OS.rows(bt.start, bt.lens)]
        rest = np.setdiff1d(np.arange(len(q_host)), rows)
        assert np.array_equal(q_host[rest].view(np.uint16), np.asarray(q_canary)[rest].view(np.uint16))
    for name, (codes, scales), (wcodes, wscales, exact) in zip("kv", got, want):
        assert np.array_equal(scales, wscales), name
        new = ~np.isnan(exact)
        if name == "v":
            same = (codes == wcodes) | ((codes & 127) == 127) & ((wcodes & 127) == 127)
            assert same.all()
            continue
        finite = np.isfinite(exact)
        bad = new & ~finite
        assert np.array_equal(codes[~new], wcodes[~new]) or ((codes[~new] & 127)[codes[~new] != wcodes[~new]] == 127).all()
        assert ((codes[bad] & 127) == 127).all()
        x = np.clip(np.where(finite, exact, 0.0), -448, 448)
        pair = np.hypot(exact[..., :64], exact[..., 64:])
        slack = 2.0**-16 * np.concatenate([pair, pair], axis=-1)
        err = np.abs(OS.e4m3_values()[codes] - x)
        assert (err[finite] <= (half_step(np.abs(x) + np.where(finite, slack, 0)) + slack)[finite]).all()
    return got


@pytest.mark.parametrize("Hq,Hkv,ps,tokens,before,kw", [
    (32, 8, 16, [1], [0], {}),
    (32, 8, 16, [1, 1, 1], [15, 16, 700], {}),
    (1, 1, 16, [5], [3], {}),
    (14, 2, 32, [3, 0, 17, 1], [31, 9, 0, 64], {"pad": 5}),
    (28, 4, 64, [66, 1], [5, 63], {"slot_major": True}),
    (40, 8, 16, [9, 40], [2, 0], {"first": 3, "pad": 2}),
    (64, 8, 256, [130], [203], {}),
    (3, 3, 16, [1] * 70, list(range(70)), {}),
    (8, 8, 16, [700], [5], {}),                                     # windows of 16 rows
    (2, 2, 16, [1, 2, 0, 3] * 600, [7, 15, 40, 30] * 600, {}),      # and many sequences in each
    (16, 8, 32, [1, 500, 1, 1, 37], [90, 17, 0, 31, 15], {"pad": 9, "first": 5}),
])
@pytest.mark.parametrize("norm", ["both", "q", "none"])
def test_append(Hq, Hkv, ps, tokens, before, kw, norm):
    say("append8", Hq, Hkv, ps, len(tokens), sum(tokens), norm)
    if norm != "both" and sum(tokens) > 200:
        pytest.skip("norms covered by the smaller cases")
    rng = np.random.default_rng(sum(tokens) + Hq + ps)
    bt = Batch8(rng, tokens, before, ps, Hkv, garbage=None, spread=3, **kw)
    width = (Hq + 2 * Hkv) * 128
    # rows of unlike magnitudes: some raise their block's scale, some do not
    wide = (rng.standard_normal((bt.T, width + 24)) * np.exp(1.5 * rng.standard_normal((bt.T, 1)))).astype(np.float16)
    qw = (1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm != "none" else None
    kw_ = (1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm == "both" else None
    cs = decode.rope_table(int(bt.lens.max()) + 1, 1e6, DEV)
    check_append(rng, bt, wide[:, :width], qw, kw_, cs, Hq, f16(rng, (bt.T, Hq, 128)))


def test_append_strided_rows():
    """Rows and page tables that are views of wider arrays."""
    say("append8 strided")
    rng = np.random.default_rng(2)
    Hq, Hkv = 6, 2
    bt = Batch8(rng, [5, 1], [9, 40], 16, Hkv, garbage=None)
    width = (Hq + 2 * Hkv) * 128
    wide = f16(rng, (bt.T, width + 40))
    cs = decode.rope_table(64, 1e6, DEV)
    k, v, ks, vs, table, start, lens = bt.device8()
    table_wide = torch.full((2, bt.table.shape[1] + 5), 77, dtype=torch.int32, device=DEV)
    table_wide[:, 2:2 + bt.table.shape[1]] = table
    laq.paged_append_e4m3(dev(wide)[:, 8:8 + width], None, None, cs, k, v, ks, vs,
                          table_wide[:, 2:2 + bt.table.shape[1]], start, lens, Hq, EPS)
    torch.cuda.synchronize()
    check_append(rng, bt, wide[:, 8:8 + width], None, None, cs, Hq, np.zeros((bt.T, Hq, 128), np.float16),
                 got=((host(k), host(ks)), (host(v), host(vs))))


def test_append_token_by_token():
    """A sequence that grows by one row a call, magnitudes rising and falling:
    every call from the caches of the one before."""
    say("append8 token by token")
    rng = np.random.default_rng(3)
    Hq, Hkv, ps = 2, 2, 32
    bt = Batch8(rng, [1], [0], ps, Hkv, spare=1, extra_columns=2, garbage=None)
    bt.table[0] = [1, 0, -1]
    cs = decode.rope_table(96, 1e6, DEV)
    for pos in range(66):  # past the pages that are there
        bt.lens[0] = pos + 1
        qkv = f16(rng, (1, (Hq + 2 * Hkv) * 128), float(np.exp(2.5 * rng.standard_normal())))
        (bt.kc, bt.ks), (bt.vc, bt.vs) = check_append(rng, bt, qkv, None, None, cs, Hq, np.zeros((1, Hq, 128), np.float16))


def test_append_scales():
    """Zeros, values at and past the borders of a scale, the largest and
    smallest fp16 numbers, infinities and NaN."""
    say("append8 scales")
    rng = np.random.default_rng(4)
    Hq, Hkv = 1, 1
    cs = torch.cat([torch.ones(64, 64), torch.zeros(64, 64)], dim=1).to(DEV).contiguous()  # no rotation
    tops = [0.0, 2.0**-24, 2.0**-14, 448 * 2.0**-15, 448 * 2.0**-14, 0.875, 1.75, 1.7509765625, 448.0, 448.25, 57344.0,
            57376.0, 65504.0, 2.0**-3 * 464, 31.0]
    for n in (1, 3):
        for top in tops:
            bt = Batch8(rng, [n, n], [0, 5], 16, Hkv, garbage=None)
            bt.ks[:], bt.vs[:] = 250, 0  # whatever the block held
            bt.ks[bt.table[1, 0]], bt.vs[bt.table[1, 0]] = 113, 90
            qkv = (f16(rng, (2 * n, 384)).astype(np.float64) / 8).astype(np.float16)
            m = np.abs(qkv.astype(np.float64)).max()
            qkv = (qkv.astype(np.float64) / m * top).astype(np.float16)
            qkv[0, 130], qkv[n, 300] = top, -top
            check_append(rng, bt, qkv, None, None, cs, Hq, np.zeros((2 * n, 1, 128), np.float16))
            bad = qkv.copy()
            bad[0, [131, 260]], bad[n, [140, 301]] = [np.inf, np.nan], [-np.inf, np.inf]
            check_append(rng, bt, bad, None, None, cs, Hq, np.zeros((2 * n, 1, 128), np.float16))


def test_append_places_that_are_not_there():
    """Positions outside the rotation table or the page table, pages outside the
    cache, negative positions: q zero or computed, nothing appended anywhere."""
    say("append8 bad places")
    rng = np.random.default_rng(11)
    Hq, Hkv, ps, P = 4, 2, 16, 3
    bt = Batch8(rng, [1], [0], ps, Hkv, spare=2, garbage=None)
    bt.table = np.array([[0, -1], [P, 1], [2, 2**31 - 1], [0, 1], [1, 1]], dtype=np.int32)
    # seq 0: position 16, page -1; 1: position 3, page P; 2: position 20, a huge page;
    # 3: position 32, past the page table; 4: two rows at positions -1 and 0 (page 1)
    bt.lens = np.array([17, 4, 21, 33, 1], dtype=np.int32)
    bt.start = np.array([0, 1, 2, 3, 4, 6], dtype=np.int32)
    bt.T = 6
    qkv = f16(rng, (6, (Hq + 2 * Hkv) * 128))
    for S in (40, 17):
        (kc, ks), (vc, vs) = check_append(rng, bt, qkv, None, None, decode.rope_table(S, 1e6, DEV), Hq,
                                          np.zeros((6, Hq, 128), np.float16))
        assert np.array_equal(kc[[0, 2]], bt.kc[[0, 2]]) and np.array_equal(ks[[0, 2]], bt.ks[[0, 2]])


@pytest.mark.parametrize("T,Hkv", [(40, 2), (1200, 8)])
def test_append_row_starts_outside_the_batch(T, Hkv):
    """Row starts below 0 and past T count as the nearer of the two; a sequence
    whose length is negative or 0 has no place for its rows."""
    say("append8 row starts", T)
    rng = np.random.default_rng(12)
    Hq = Hkv
    bt = Batch8(rng, [T // 4] * 4, [3, 30, 17, 0], 16, Hkv, garbage=None)
    qkv = f16(rng, (T, (Hq + 2 * Hkv) * 128))
    cs = decode.rope_table(T + 64, 1e6, DEV)
    q0 = f16(rng, (T, Hq, 128))
    inside = bt.start.copy()
    k, v, ks, vs, table, start, lens = bt.device8()
    start[0], start[4] = -50, T + 1000
    q = laq.paged_append_e4m3(dev(qkv), None, None, cs, k, v, ks, vs, table, start, lens, Hq, EPS, q_out=dev(q0))
    torch.cuda.synchronize()
    bt.start = inside
    check_append(rng, bt, qkv, None, None, cs, Hq, q0, got=((host(k), host(ks)), (host(v), host(vs))))
    bt.lens[:] = [0, -5, 1, T // 4 - 2]
    check_append(rng, bt, qkv, None, None, cs, Hq, q0)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def small(bt, Hq):
    """Whether each sequence's probabilities are two fp16 numbers (else one, where sizes choose the larger kernel)."""
    R = Hq // bt.Hkv
    few = bt.T * R <= 16 * len(bt.tokens)
    return [few or n * R <= 16 for n in bt.tokens]


def check_rows(bt, Hq, q, got, window, canary):
    ref, weight, reach = OS.paged_attention(q, bt.k, bt.v, bt.table, bt.start, bt.lens, window, canary)
    few = small(bt, Hq)
    for b in range(len(bt.tokens)):
        mine = slice(int(bt.start[b]), int(bt.start[b + 1]))
        if few[b]:  # (2^-20 of the weights, with the output's own rounding)
            attention_check(got[mine], ref[mine], weight[mine] * (1 + 2.0**-7), reach[mine] + 2.0, int(bt.lens.max()), False)
        else:
            attention_check(got[mine], ref[mine], weight[mine], reach[mine], int(bt.lens.max()), True)
    other = np.ones(bt.T, dtype=bool)
    other[bt.start[0]:bt.start[-1]] = False
    assert np.array_equal(got[other], canary[other])


def attend(bt, q, window=0, out=None):
    got = laq.paged_attention_e4m3(dev(q), *bt.device8(), window=window, out=out)
    torch.cuda.synchronize()
    return got.cpu().numpy()


def run_attention(rng, bt, Hq, window=0, q_scale=1.5, check=True):
    q = f16(rng, (bt.T, Hq, 128), q_scale)
    canary = f16(rng, (bt.T, Hq, 128))
    got = attend(bt, q, window, dev(canary))
    if check:
        check_rows(bt, Hq, q, got, window, canary)
    return q, got


@pytest.mark.parametrize("few", [True, False])
def test_attention_every_code_and_scale(few):
    """A row that sees one position returns its value: every code under every
    scale, and scales outside the range as its borders.  And as a key: scores of
    single dimensions order two positions alike."""
    say("attention8 codes", few)
    rng = np.random.default_rng(1)
    scales = list(range(112, 135)) + [0, 111, 135, 255]
    n = len(scales)
    tokens = [1] * n if few else [1] * n + [200]
    bt = Batch8(rng, tokens, [0] * len(tokens), 16, 2)
    for i, s in enumerate(scales):
        for g in range(2):
            bt.vc[bt.table[i, 0], g, 0] = np.arange(128) + 128 * g
            bt.vs[bt.table[i, 0], g] = s
    q = f16(rng, (bt.T, 2, 128))
    bt.values()
    got = attend(bt, q)
    for i in range(n):
        want = bt.v[bt.table[i, 0], :, 0]
        assert np.array_equal(np.isnan(got[i]), np.isnan(want))
        fine = ~np.isnan(want)
        assert np.array_equal(got[i][fine], want[fine]), scales[i]


@pytest.mark.parametrize("tokens,before,Hq,Hkv,kw", [
    ([1, 1], [50, 61], 8, 2, {}),
    ([1], [2100], 16, 2, {}),                              # split over ranges of positions
    ([1, 1, 150, 1, 2], [33, 60, 20, 47, 40], 8, 2, {}),   # decoding rows beside a chunk
    ([1, 1], [50, 61], 8, 2, {"pad": 60}),                 # decoding rows of a batch with padding
    ([4], [44], 4, 1, {"pad": 1}),                         # 16 query rows
])
def test_attention_of_few_rows_keeps_22_bits(tokens, before, Hq, Hkv, kw):
    """Sequences of up to 16 query rows a key/value head, whatever stands beside
    them: probabilities are not rounded to 16 bits.

    Scores are small sums of four products and values are +1 and -1, as many of
    the one as of the other, so that outputs are near 0 and their own fp16
    rounding is small.  The bound, relative to the weights' sum of |v| = 1: scores
    are fp32 sums (136 x 2^-24 of the sum of magnitudes, in a weight and in the
    denominator), L x 2^-24 in the value sums and in the denominator, 2^-20 of a
    probability cut off (2^-10 of its first part's remainder, itself below 2^-10),
    and the rounding of the output, 2^-11 of it."""
    say("few rows8", tokens, Hq, kw)
    rng = np.random.default_rng(sum(tokens) + sum(before) + Hq)
    bt = Batch8(rng, tokens, before, 16, Hkv, **kw)
    bt.vs[:] = 127
    for b, n in enumerate(bt.lens):
        for g in range(Hkv):
            signs = np.array([rng.permutation(np.resize([0x38, 0xB8], n)) for _ in range(128)])
            for t in range(n):
                bt.vc[bt.table[b, t // 16], g, t % 16] = signs[:, t]
    bt.values()
    q = np.zeros((bt.T, Hq, 128), dtype=np.float16)
    q[..., 5::32] = f16(rng, (bt.T, Hq, 4), 0.5)
    got = attend(bt, q).astype(np.float64)
    ref, weight, reach = OS.paged_attention(q, bt.k, bt.v, bt.table, bt.start, bt.lens, 0, np.zeros_like(got))
    few = small(bt, Hq)
    mine = [(r, pos) for r, b, pos in OS.rows(bt.start, bt.lens) if few[b]]
    rows = [r for r, _ in mine]
    assert len(rows) >= 1 and np.allclose(weight[rows], 1)
    L = np.array([pos + 1 for _, pos in mine])[:, None, None]
    tol = 2.0**-11 * np.abs(ref[rows]) + 2 * 136 * 2.0**-24 * reach[rows][..., None] + 2 * L * 2.0**-24 + 2.0**-20 + 2.0**-25
    err = np.abs(got[rows] - ref[rows])
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("tokens,before", [([1, 1], [60, 1500]), ([40], [90]), ([300, 1], [50, 700])])
def test_attention_huge_scores(tokens, before):
    """Scores from 2^20 on, some a few steps of 32 bits apart: all values are 1, so
    that outputs are 1 whatever the weights (each probability's rounding 2^-11 of
    it, the output's 2^-11, sums over L positions 2 L x 2^-24)."""
    say("huge scores8", tokens)
    rng = np.random.default_rng(5 + sum(tokens))
    bt = Batch8(rng, tokens, before, 16, 2)
    bt.ks[:] = rng.choice([126, 131, 134], bt.ks.shape)
    bt.vs[:] = 127
    bt.vc[np.broadcast_to(bt.used[:, None], bt.vc.shape[:3])] = 0x38
    q = f16(rng, (bt.T, 4, 128), 2000.0)
    got = attend(bt, q)
    mine = slice(bt.start[0], bt.start[-1])
    tol = 2 * 2.0**-11 + 2 * int(bt.lens.max()) * 2.0**-24
    assert (np.abs(got[mine].astype(np.float64) - 1) <= tol).all()


CASES = [
    # decoding: one row a sequence, lengths around steps, blocks and ranges
    (32, 8, 16, [1], [0], 0, {}),
    (32, 8, 16, [1], [31], 0, {}),
    (32, 8, 16, [1], [32], 0, {}),
    (32, 8, 32, [1, 1, 1, 1], [0, 127, 128, 129], 0, {}),
    (8, 1, 64, [1, 1], [1000, 5], 0, {}),
    (5, 5, 16, [1], [255], 0, {}),
    (64, 8, 16, [1, 1, 1], [256, 300, 2047], 0, {"pad": 3}),
    (16, 1, 128, [1], [700], 0, {}),
    (48, 2, 16, [1, 1], [90, 300], 0, {}),       # 24 heads a key/value head: two tiles
    (14, 2, 16, [2, 1, 2], [500, 90, 33], 0, {}),  # seven
    (8, 8, 16, [1] * 70, [3 * i for i in range(70)], 0, {}),
    (4, 4, 16, [3, 0, 1], [40, 77, 0], 0, {"first": 2, "pad": 1}),
    (32, 8, 16, [1, 1], [600, 100], 64, {}),
    (32, 8, 16, [1], [1500], 1, {}),
    (8, 2, 16, [4, 4], [300, 5], 33, {}),
    (4, 1, 32, [1], [9000], 0, {"slot_major": True}),  # more than 32 steps a wave
    # chunks
    (32, 8, 16, [16], [0], 0, {}),
    (32, 8, 16, [33], [100], 0, {}),
    (4, 4, 64, [64], [0], 0, {}),
    (4, 4, 64, [65], [63], 0, {}),
    (2, 1, 16, [200], [1], 0, {}),
    (10, 2, 16, [70, 1, 0, 20], [130, 600, 50, 0], 0, {"pad": 7, "first": 1}),
    (1, 1, 16, [129, 127], [0, 512], 0, {"slot_major": True}),
    (8, 1, 256, [40, 1], [500, 1200], 0, {}),
    (6, 2, 16, [90], [200], 40, {}),
    (6, 2, 32, [90, 30], [200, 5], 128, {"slot_major": True}),
    (24, 1, 16, [30], [77], 0, {}),
    (2, 1, 16, [300, 1], [1700, 1500], 0, {}),   # more than 16 tiles
]


@pytest.mark.parametrize("Hq,Hkv,ps,tokens,before,window,kw", CASES)
def test_attention(Hq, Hkv, ps, tokens, before, window, kw):
    say("attention8", Hq, Hkv, ps, len(tokens), sum(tokens), max(before), window)
    rng = np.random.default_rng(sum(tokens) * 7 + sum(before) + Hq + window)
    bt = Batch8(rng, tokens, before, ps, Hkv, **kw)
    if window:  # pages that no row sees were given back
        for b, p in enumerate(before):
            bt.table[b, :max(0, p - window + 1) // ps] = -1
    q, got = run_attention(rng, bt, Hq, window)
    again = attend(bt, q, window)  # the same on every call
    mine = slice(bt.start[0], bt.start[-1])
    assert np.array_equal(again[mine].view(np.uint16), got[mine].view(np.uint16))


@pytest.mark.parametrize("tokens,before", [([1, 1], [90, 60]), ([40, 30], [90, 40])])
def test_attention_extreme_scales(tokens, before):
    """Blocks under the smallest and the largest scales beside each other: the
    values are what the codes stand for, in both products."""
    say("attention8 extreme scales", tokens)
    rng = np.random.default_rng(15)
    bt = Batch8(rng, tokens, before, 16, 2)
    bt.vs[:] = rng.choice([112, 113, 127, 133, 134], bt.vs.shape)
    bt.ks[:] = rng.choice([112, 116, 118, 119], bt.ks.shape)
    bt.values()
    run_attention(rng, bt, 4)


@pytest.mark.parametrize("Hq,tokens", [(2, [1, 1]), (2, [80, 3])])
def test_attention_large_scores(Hq, tokens):
    """Scores of several hundred, the largest first, last and in the middle."""
    say("attention8 large scores", tokens)
    rng = np.random.default_rng(8)
    bt = Batch8(rng, tokens, [300, 130], 16, 1)
    for t in (0, 150, 299):
        bt.kc[bt.table[0, t // 16], 0, t % 16] = 126
    bt.ks[:] = 121
    bt.values()
    run_attention(rng, bt, Hq, q_scale=8.0)


@pytest.mark.parametrize("tokens,before,window", [([1, 1], [100, 60], 0), ([4, 2], [90, 40], 48), ([70, 40], [90, 40], 0),
                                                  ([70, 40], [90, 40], 50), ([60, 2], [90, 40], 0)])
def test_attention_unseen_values(tokens, before, window):
    """NaN among positions that a row does not see, keys and values, leave the
    row as it is; a row that sees one is NaN there."""
    say("attention8 unseen", tokens, window)
    rng = np.random.default_rng(21)
    Hq, Hkv, ps = 4, 2, 16
    bt = Batch8(rng, tokens, before, ps, Hkv)
    q, clean = run_attention(rng, bt, Hq, window)
    for b in range(2):
        at = bt.lens[b] - 1 - (tokens[b] // 2 if tokens[b] > 1 else 0)  # a position that later rows alone see
        pg, sl = bt.table[b, at // ps], at % ps
        first = max(0, before[b] - window + 1) if window else 0
        for code in (0x7F, 0xFF):
            saved = bt.kc.copy(), bt.vc.copy()
            bt.vc[pg, 1, sl, ::3] = code
            bt.kc[pg, 0, sl, 5] = code
            if window and first > 0:  # and one before every window
                bt.vc[bt.table[b, (first - 1) // ps], 0, (first - 1) % ps] = code
            out = attend(bt, q, window)
            bt.kc, bt.vc = saved
            for r, s, pos in OS.rows(bt.start, bt.lens):
                sees = s == b and pos >= at and (not window or pos - at < window)
                if not sees:
                    assert np.array_equal(out[r].view(np.uint16), clean[r].view(np.uint16)), (r, pos, code)
                else:
                    assert np.isnan(out[r, 2:, ::3]).all() and np.isnan(out[r, :2]).all()
                    assert np.array_equal(out[r, 2:, 1::3].view(np.uint16), clean[r, 2:, 1::3].view(np.uint16))


@pytest.mark.parametrize("tokens", [[1, 1, 2], [40, 30, 9], [40, 1, 2]])
def test_attention_rows_that_see_nothing(tokens):
    """No page of the sequence is there, the sequence has fewer positions than
    rows, its positions lie past the page table: zeros where nothing is seen."""
    say("attention8 nothing seen", tokens)
    rng = np.random.default_rng(33)
    bt = Batch8(rng, tokens, [50, 20, 0], 16, 2)
    bt.table[0] = [-1, bt.P, 2**31 - 1, -2**31, -1, -7][:bt.table.shape[1]] + [-1] * (bt.table.shape[1] - 6)
    bt.lens[2] -= tokens[2] // 2 + 1 if tokens[2] > 1 else 0  # the first rows have negative positions
    q, got = run_attention(rng, bt, 4)
    assert not got[:tokens[0]].any()
    bt.lens[1] = bt.table.shape[1] * 16 + 500  # positions past the table
    bt.table[1] = bt.table[1, 0]
    q, got = run_attention(rng, bt, 4, check=False)
    assert np.isfinite(got[:tokens[0]]).all()
    bt.lens[:] = 0
    q, got = run_attention(rng, bt, 4, check=False)
    assert not got.any()


def test_attention_missing_pages_inside():
    """A page given back in the middle of a sequence is skipped."""
    say("attention8 missing pages")
    rng = np.random.default_rng(4)
    for tokens, Hq in (([1, 1], 8), ([50, 20], 8), ([1], 2)):
        bt = Batch8(rng, tokens, [200, 90][:len(tokens)], 16, 2)
        bt.table[0, 3] = -1
        bt.table[0, 6] = bt.P + 5
        if len(tokens) > 1:
            bt.table[1, 0] = -1
        run_attention(rng, bt, Hq)


@pytest.mark.parametrize("tokens,before,Hq,Hkv,ps,window", [
    ([255, 1, 0, 3], [1500, 300, 0, 1000], 1, 1, 16, 0),
    ([257, 2], [1800, 1023], 1, 1, 16, 0),
    ([300, 5], [2300, 1100], 2, 1, 64, 1100),
    ([5] * 40 + [300] + [5] * 30, [20] * 40 + [1500] + [100] * 30, 4, 2, 16, 0),
])
def test_attention_chunks_over_many_tiles(tokens, before, Hq, Hkv, ps, window):
    """Chunks of several blocks of rows over more positions than one set of page
    offsets and scales covers (1024), pages missing around its ends, NaN among
    the values that some rows of a block do not see."""
    say("attention8 many tiles", tokens[:4], Hq, Hkv, window)
    rng = np.random.default_rng(len(tokens) + Hq + ps)
    bt = Batch8(rng, tokens, before, ps, Hkv)
    long = int(np.argmax(bt.lens))
    for at in (1000, 1023, 1024, 2040, 2064):
        if at < bt.lens[long]:
            bt.table[long, at // ps] = -1 if at != 1024 else bt.P
    q, clean = run_attention(rng, bt, Hq, window)
    at = int(bt.lens[long]) - 2  # the last two rows see it
    bt.vc[bt.table[long, at // ps], 0, at % ps, ::5] = 0xFF
    out = attend(bt, q, window)
    R = Hq // Hkv
    for r, b, pos in OS.rows(bt.start, bt.lens):
        if b == long and pos >= at:
            assert np.isnan(out[r, :R, ::5]).all()
            out[r, :R, ::5] = clean[r, :R, ::5]
    assert np.array_equal(out.view(np.uint16), clean.view(np.uint16))


@pytest.mark.parametrize("window", [0, 300])
def test_attention_large_batches(window):
    """As many query rows as the kernel of 256 rows a block takes: chunks beside a
    decoding sequence, missing pages, NaN among values that some rows do not see.
    Some rows of every sequence against 64 bits."""
    say("attention8 large", window)
    rng = np.random.default_rng(40 + window)
    Hq, Hkv, ps, tokens, before = 64, 8, 32, [1500, 1, 600], [100, 1700, 700]
    bt = Batch8(rng, tokens, before, ps, Hkv, pad=5)
    bt.table[2, [3, 30]] = [-1, bt.P]
    seen_by_few = int(bt.lens[0]) - 3
    bt.vc[bt.table[0, seen_by_few // ps], 1, seen_by_few % ps, ::7] = 0x7F
    bt.values()
    assert bt.T * Hq >= 512 * 256
    q = f16(rng, (bt.T, Hq, 128))
    canary = f16(rng, (bt.T, Hq, 128))
    got = attend(bt, q, window, dev(canary))
    again = attend(bt, q, window, dev(canary))
    assert np.array_equal(got.view(np.uint16), again.view(np.uint16))
    assert np.array_equal(got[-5:], canary[-5:])
    rows = [(r, b, pos) for r, b, pos in OS.rows(bt.start, bt.lens)]
    picked = [rows[i] for i in sorted(set(rng.integers(0, len(rows), 40).tolist()) |
                                      {0, 1, 31, 32, 255, 256, 1496, 1497, 1499, 1500, 1501, len(rows) - 1})]
    few = small(bt, Hq)
    for r, b, pos in picked:
        t = np.arange(max(0, pos - window + 1) if window else 0, pos + 1)
        pages = bt.table[b, t // ps]
        t, pages = t[(pages >= 0) & (pages < bt.P)], pages[(pages >= 0) & (pages < bt.P)]
        for g in range(Hkv):
            K, V = (c[pages, g, t % ps].astype(np.float64) for c in (bt.k, bt.v))
            x = q[r, 8 * g:8 * g + 8].astype(np.float64)
            s = x @ K.T / 128**0.5
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            out, nan = got[r, 8 * g:8 * g + 8], np.isnan(V).any(0)
            assert np.isnan(out[:, nan]).all()
            V = np.where(nan, 0.0, V)
            reach = (np.abs(x) @ np.abs(K).T).max(1) / 128**0.5
            attention_check(np.where(nan, np.float16(0), out), p @ V, p @ np.abs(V), reach + 2.0, len(t), not few[b])


@pytest.mark.parametrize("tokens,before,kw", [([1, 1], [2999, 40000], {}), ([40], [6000], {}), ([1] * 80, [700] * 80, {}),
                                              ([150, 1, 1], [3000, 5000, 20], {"pad": 2})])
def test_attention_is_that_of_the_values(tokens, before, kw):
    """Many ranges per sequence, many sequences: the attention over an fp16
    cache of the same values, within both tolerances."""
    say("attention8 of values", tokens[:3], before[:3])
    rng = np.random.default_rng(len(tokens))
    Hq, Hkv = 8, 2
    bt = Batch8(rng, tokens, before, 64, Hkv, **kw)
    q = f16(rng, (bt.T, Hq, 128))
    got = attend(bt, q).astype(np.float64)
    bt.k[~bt.used[:, None].repeat(Hkv, 1)] = 0
    bt.v[~bt.used[:, None].repeat(Hkv, 1)] = 0
    ref = laq.paged_attention(dev(q), dev(bt.k), dev(bt.v), dev(bt.table), dev(bt.start), dev(bt.lens))
    ref = ref.cpu().numpy().astype(np.float64)
    mine = slice(bt.start[0], bt.start[-1])
    # outputs are means of values of magnitude up to 4: roundings of both to fp16, of both's probabilities
    # (2^-11 of |v|, of which a mean of the weights' errors remains), sums over L positions in 32 bits
    size = np.abs(bt.v.astype(np.float64)).max()
    tol = 2.0**-10 * np.abs(ref[mine]) + 2 * 2.0**-11 * size + 4 * bt.lens.max() * 2.0**-24 * size
    assert (np.abs(got[mine] - ref[mine]) <= tol).all()


def test_far_pages():
    """Pages past 2^31 bytes of the cache, and a scale table of their size; the
    other pages are never read."""
    say("far pages8")
    rng = np.random.default_rng(6)
    Hq, Hkv, ps = 4, 2, 64
    P = 2**32 // (Hkv * ps * 128) + 40
    k, v = (torch.empty((P, Hkv, ps, 128), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.empty((P, Hkv, ps // 16), dtype=torch.uint8, device=DEV).view(E8M0) for _ in range(2))
    bt = Batch8(rng, [1, 30], [200, 100], ps, Hkv)
    far = P - bt.P
    table = np.where(bt.table >= 0, bt.table + far, -1).astype(np.int32)
    near = bt.device8()
    for a, b in zip((k, v, ks, vs), near):
        a.view(torch.uint8)[far:] = b.view(torch.uint8)
    q = f16(rng, (bt.T, Hq, 128))
    rest = (dev(table), dev(bt.start), dev(bt.lens))
    out = laq.paged_attention_e4m3(dev(q), k, v, ks, vs, *rest)
    assert torch.equal(out, laq.paged_attention_e4m3(dev(q), *near))
    qkv = dev(f16(rng, (bt.T, (Hq + 2 * Hkv) * 128)))
    cs = decode.rope_table(300, 1e6, DEV)
    laq.paged_append_e4m3(qkv, None, None, cs, k, v, ks, vs, *rest, Hq, EPS)
    laq.paged_append_e4m3(qkv, None, None, cs, *near, Hq, EPS)
    torch.cuda.synchronize()
    for a, b in zip((k, v, ks, vs), near):
        assert torch.equal(a.view(torch.uint8)[far:], b.view(torch.uint8))


def test_shared_pages():
    """Sequences with the same pages in front (a shared prompt), the same sequence
    twice, and appends behind the shared pages: as with pages of their own."""
    say("shared pages8")
    rng = np.random.default_rng(31)
    Hq, Hkv, ps = 8, 2, 16
    for tokens, before in (([1, 1, 1], [80, 83, 95]), ([20, 1, 33], [64, 70, 66])):
        bt = Batch8(rng, tokens, before, ps, Hkv)
        for b in (1, 2):  # the first four pages of all hold the same
            for x in (bt.kc, bt.vc, bt.ks, bt.vs):
                x[bt.table[b, :4]] = x[bt.table[0, :4]]
        bt.values()
        own = bt.device8()
        table = bt.table.copy()
        table[1:, :4] = table[0, :4]
        shared = own[:4] + (dev(table),) + own[5:]
        shared = tuple(t.clone() for t in shared)
        qkv = dev(f16(rng, (bt.T, (Hq + 2 * Hkv) * 128)))
        cs = decode.rope_table(300, 1e6, DEV)
        outs = []
        for d in (own, shared):
            q = laq.paged_append_e4m3(qkv, None, None, cs, *d, Hq, EPS)
            outs.append((q, laq.paged_attention_e4m3(q, *d)))
        torch.cuda.synchronize()
        for x, y in zip(*outs):
            assert torch.equal(x, y)
        for x, y in zip(own[:4], shared[:4]):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # one sequence's new row as two sequences of a batch
    bt = Batch8(rng, [1], [700], ps, Hkv)
    q = f16(rng, (1, Hq, 128))
    kc, vc, ks, vs, table, _, lens = bt.device8()
    twice = laq.paged_attention_e4m3(dev(np.repeat(q, 2, 0)), kc, vc, ks, vs, table.repeat(2, 1), dev(np.array([0, 1, 2], np.int32)),
                                     lens.expand(2).contiguous())
    assert torch.equal(twice[0], twice[1])
    once = attend(bt, q)[0].astype(np.float64)
    # (ranges may differ: both outputs' roundings, 2^-20 of |v| cut off each, sums over 701 positions in 32 bits)
    size = np.abs(bt.v.transpose(0, 2, 1, 3)[bt.used].astype(np.float64)).max()
    tol = 2.0**-10 * np.abs(once) + 2 * size * 2.0**-20 + 4 * 701 * 2.0**-24 * size
    assert (np.abs(twice[0].cpu().numpy().astype(np.float64) - once) <= tol).all()


def test_in_a_graph():
    """Append and attention captured once; the replays follow the arrays that
    change between them."""
    say("graph8")
    rng = np.random.default_rng(14)
    Hq, Hkv, ps, B, width = 8, 2, 16, 3, 40
    P = B * width
    table = dev(rng.permutation(P).astype(np.int32).reshape(B, width))
    start = dev(np.array([0, 1, 2, 3], dtype=np.int32))
    cs = decode.rope_table(width * ps, 1e6, DEV)
    runs = []
    for graphed in (False, True):
        gen = np.random.default_rng(15)
        k, v = (torch.zeros((P, Hkv, ps, 128), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
        ks, vs = (torch.zeros((P, Hkv, ps // 16), dtype=torch.uint8, device=DEV).view(E8M0) for _ in range(2))
        lens = dev(np.array([1, 1, 1], dtype=np.int32))
        qkv = torch.zeros((B, (Hq + 2 * Hkv) * 128), dtype=torch.float16, device=DEV)
        q = torch.zeros((B, Hq, 128), dtype=torch.float16, device=DEV)
        out = torch.zeros_like(q)
        ws = torch.empty(max(laq.paged_attention_e4m3_workspace_bytes(B, B, Hq, Hkv, width * ps), 16), dtype=torch.uint8, device=DEV)

        def step():
            laq.paged_append_e4m3(qkv, None, None, cs, k, v, ks, vs, table, start, lens, Hq, EPS, q_out=q)
            laq.paged_attention_e4m3(q, k, v, ks, vs, table, start, lens, out=out, workspace=ws)
        got, g = [], None
        for i, grown in enumerate((1, 1, 40, 1, 300, 1, 200)):
            lens += grown if i else 0
            qkv.copy_(dev(f16(gen, qkv.shape, 1.0 + i)))
            if graphed and i == 1:
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                saved = [t.clone() for t in (k.view(torch.uint8), v.view(torch.uint8), ks.view(torch.uint8), vs.view(torch.uint8))]
                with torch.cuda.graph(g):
                    step()
                for t, s in zip((k, v, ks, vs), saved):
                    t.view(torch.uint8).copy_(s)
            if g is not None:
                g.replay()
            else:
                step()
            torch.cuda.synchronize()
            got.append([t.clone() for t in (out.view(torch.int16), k.view(torch.uint8), v.view(torch.uint8),
                                            ks.view(torch.uint8), vs.view(torch.uint8))])
        runs.append(got)
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_streams_at_once():
    """Two batches on two streams, each with its own workspace, while the
    current stream is a third: what each gives alone."""
    say("two streams8")
    rng = np.random.default_rng(16)
    Hq, Hkv = 8, 2
    sets, alone = [], []
    for tokens, before in (([1, 1], [3000, 700]), ([90], [500])):
        bt = Batch8(rng, tokens, before, 16, Hkv)
        q = dev(f16(rng, (bt.T, Hq, 128)))
        d = bt.device8()
        nbytes = laq.paged_attention_e4m3_workspace_bytes(len(tokens), bt.T, Hq, Hkv, d[4].shape[1] * 16)
        sets.append((q, d, torch.empty(nbytes, dtype=torch.uint8, device=DEV), torch.zeros_like(q)))
        alone.append(laq.paged_attention_e4m3(q, *d))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, (q, d, ws, out) in zip(streams, sets):
            with torch.cuda.stream(s):
                laq.paged_attention_e4m3(q, *d, out=out, workspace=ws)
    torch.cuda.synchronize()
    for (_, _, _, out), ref in zip(sets, alone):
        assert torch.equal(out, ref)


# ---------------------------------------------------------------------------
# logits before sampling
# ---------------------------------------------------------------------------
def adjust_case(rng, R, V, H, N, mask, prompt=True):
    logits = (3 * rng.standard_normal((R, V)) - 1).astype(np.float16)
    history = rng.integers(-3, V + 3, (R, H)).astype(np.int32) if H else None
    a = dict(history=history)
    if H:
        history[:, ::3] = rng.integers(0, min(V, 9), history[:, ::3].shape)  # repeated ones
        n = rng.integers(-2, H + 4, R).astype(np.int32)
        n[0] = H
        a.update(history_len=n, prompt_len=rng.integers(-1, H + 2, R).astype(np.int32) if prompt else None,
                 repetition=(0.7 + rng.random(R)).astype(np.float32), frequency=(rng.random(R) - 0.3).astype(np.float32),
                 presence=(rng.random(R) - 0.3).astype(np.float32))
    if N:
        t = rng.integers(-2, V + 2, (R, N)).astype(np.int32)
        t[:, N // 2:] = t[:, :N - N // 2]  # listed twice
        val = (4 * rng.standard_normal((R, N))).astype(np.float32)
        val[:, 0] = -np.inf
        a.update(bias_token=t, bias_value=val)
    if mask:
        w = rng.integers(0, 2**32, (R, (V + 31) // 32), dtype=np.uint32)
        w[:, ::5] = 0xFFFFFFFF
        a["mask"] = w
    return logits, a


def adjust_check(logits, a, got):
    for r in range(logits.shape[0]):
        has = a.get("history") is not None
        n = min(max(int(a["history_len"][r]), 0), a["history"].shape[1]) if has else 0
        get = lambda name, off: off if a.get(name) is None else a[name][r]  # noqa: E731
        steps = {k: float(get(k, o)) for k, o in (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0))}
        told = a["history"][r, :n].tolist() if has else []
        biases = list(zip(a["bias_token"][r].tolist(), a["bias_value"][r].tolist())) if a.get("bias_token") is not None else []
        mask = a["mask"][r] if a.get("mask") is not None else None
        want = OS.adjust_row(logits[r], told, int(get("prompt_len", 0)), **steps, biases=biases, mask=mask)
        x = got[r].astype(np.float64)
        # fp32 roundings of what the sum passes through
        size = np.abs(logits[r].astype(np.float64)) * max(1, steps["repetition"], 1 / steps["repetition"])
        size = size + len(told) * abs(steps["frequency"]) + abs(steps["presence"]) + max([abs(v) for _, v in biases if np.isfinite(v)] + [0])
        inf = ~np.isfinite(want)
        assert np.array_equal(x[inf], want[inf])
        fine = ~inf
        assert (np.abs(x[fine] - want[fine]) <= (2.0**-11 * np.abs(want) + 6 * 2.0**-24 * size + 2.0**-25)[fine]).all(), r


def to_dev(a):
    return {k: None if v is None else dev(v.view(np.int32) if v.dtype == np.uint32 else v) for k, v in a.items()}


@pytest.mark.parametrize("R,V,H,N,mask", [
    (1, 1, 1, 0, False), (1, 7, 3, 2, True), (3, 8, 0, 5, True), (2, 33, 40, 0, True), (5, 2047, 17, 3, False),
    (4, 2048, 0, 0, True), (3, 2056, 100, 2047, True), (2, 8191, 5000, 10, True), (7, 8193, 900, 0, True),
    (1, 20000, 20001, 7, True), (2, 70001, 17000, 300, True), (300, 7001, 64, 4, True), (2, 32769, 16385, 0, False),
])
def test_adjust(R, V, H, N, mask):
    say("adjust", R, V, H, N, mask)
    rng = np.random.default_rng(R + V + H + N)
    logits, a = adjust_case(rng, R, V, H, N, mask, prompt=V % 2 == 1)
    got = laq.adjust_logits(dev(logits), **to_dev(a))
    torch.cuda.synchronize()
    adjust_check(logits, a, got.cpu().numpy())
    # strided rows of another alignment, and in place: the same bits, nothing beside them
    wide, wide_out = (torch.full((R, V + 13), 7.0, dtype=torch.float16, device=DEV) for _ in range(2))
    wide[:, 3:3 + V] = dev(logits)
    laq.adjust_logits(wide[:, 3:3 + V], **to_dev(a), out=wide_out[:, 6:6 + V])
    there = laq.adjust_logits(wide[:, 3:3 + V], **to_dev(a), out=wide[:, 3:3 + V])
    torch.cuda.synchronize()
    for t, o in ((wide, 3), (wide_out, 6)):
        assert torch.equal(t[:, o:o + V].view(torch.int16), got.view(torch.int16))
        assert bool((t[:, :o] == 7).all()) and bool((t[:, o + V:] == 7).all())
    assert there.data_ptr() == wide[:, 3:].data_ptr()


def test_adjust_parts():
    """Each part alone; a history of one token many times; shared histories,
    biases and masks (expanded rows); nothing at all copies, whatever the logits
    hold."""
    say("adjust parts")
    rng = np.random.default_rng(5)
    R, V = 4, 5000
    logits = f16(rng, (R, V), 4.0)
    logits[0, :4] = [np.nan, np.inf, -np.inf, -0.0]
    one = laq.adjust_logits(dev(logits))
    assert np.array_equal(one.cpu().numpy().view(np.uint16), logits.view(np.uint16))
    fine = f16(rng, (R, V), 4.0)
    ones = np.ones(R, dtype=np.float32)
    same = np.full((R, 100000), 17, dtype=np.int32)
    full = np.full(R, 100000, dtype=np.int32)
    for part in (dict(repetition=ones * 1.3), dict(frequency=ones * 1e-4), dict(presence=ones * 0.5), dict()):
        a = dict(history=same, history_len=full, **part)
        got = laq.adjust_logits(dev(fine), **to_dev(a)).cpu().numpy()
        a = {**dict(repetition=ones, frequency=ones * 0, presence=ones * 0), **a}
        adjust_check(fine, a, got)
    h, b, v, m = (rng.integers(0, V, (1, 50)).astype(np.int32), rng.integers(0, V, (1, 9)).astype(np.int32),
                  rng.standard_normal((1, 9)).astype(np.float32), rng.integers(0, 2**32, (1, (V + 31) // 32), dtype=np.uint32))
    a = dict(history=h, history_len=np.array([0, 1, 50, 20], dtype=np.int32), prompt_len=None, repetition=ones * 1.1,
             frequency=None, presence=None, bias_token=b, bias_value=v, mask=m)
    d = to_dev(a)
    for n in ("history", "bias_token", "bias_value", "mask"):
        d[n] = d[n].expand(R, -1)
    got = laq.adjust_logits(dev(fine), **d).cpu().numpy()
    for n in ("history", "bias_token", "bias_value", "mask"):
        a[n] = a[n].repeat(R, axis=0)
    adjust_check(fine, a, got)
    # logits that are infinite stay so; a mask that leaves nothing leaves -inf
    a = dict(mask=np.zeros((R, (V + 31) // 32), dtype=np.uint32))
    got = laq.adjust_logits(dev(logits), **to_dev(a)).cpu().numpy()
    assert (got == -np.inf).all()
    tok, prob = laq.sample(dev(got), dev(np.zeros(R, dtype=np.float32)))
    assert bool((tok == -1).all()) and not prob.any()


def test_adjust_far_rows():
    """Rows that begin past 2^32 elements, in place and from there to others, and
    more rows than 2^16."""
    say("adjust far rows")
    rng = np.random.default_rng(9)
    R, V, stride = 3, 4001, 2**31 + 24
    logits, a = adjust_case(rng, R, V, 200, 5, True)
    want = laq.adjust_logits(dev(logits), **to_dev(a))
    far = torch.empty(2 * stride + V, dtype=torch.float16, device=DEV).as_strided((R, V), (stride, 1))
    near = torch.zeros((R, V), dtype=torch.float16, device=DEV)
    far.copy_(dev(logits))
    laq.adjust_logits(far, **to_dev(a), out=near)
    laq.adjust_logits(far, **to_dev(a), out=far)
    torch.cuda.synchronize()
    assert torch.equal(near.view(torch.int16), want.view(torch.int16))
    assert torch.equal(far.contiguous().view(torch.int16), want.view(torch.int16))
    del far
    R, V = 70001, 3
    logits, a = adjust_case(rng, R, V, 6, 2, True)
    got = laq.adjust_logits(dev(logits), **to_dev(a)).cpu().numpy()
    picked = np.unique(np.concatenate([rng.integers(0, R, 300), [0, 65535, 65536, R - 1]]))
    adjust_check(logits[picked], {k: None if v is None else v[picked] for k, v in a.items()}, got[picked])


def test_adjust_on_two_streams():
    """Two calls at once, each on a stream of its own: what each gives alone."""
    say("adjust two streams")
    rng = np.random.default_rng(10)
    sets = []
    for R, V, H in ((5, 20001, 900), (40, 3000, 50)):
        logits, a = adjust_case(rng, R, V, H, 7, True)
        x, d = dev(logits), to_dev(a)
        sets.append((x, d, torch.zeros_like(x), laq.adjust_logits(x, **d)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, (x, d, out, _) in zip(streams, sets):
            with torch.cuda.stream(s):
                laq.adjust_logits(x, **d, out=out)
    torch.cuda.synchronize()
    for _, _, out, want in sets:
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))


def test_adjust_in_a_graph():
    """Replays follow the history, its length and the mask."""
    say("adjust graph")
    rng = np.random.default_rng(7)
    R, V, H = 3, 3001, 64
    logits, a = adjust_case(rng, R, V, H, 4, True)
    d = to_dev(a)
    x = dev(logits)
    out = torch.zeros_like(x)
    laq.adjust_logits(x, **d, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        laq.adjust_logits(x, **d, out=out)
    for i in range(4):
        logits, a = adjust_case(rng, R, V, H, 4, True)
        x.copy_(dev(logits))
        for n, t in to_dev(a).items():
            d[n].copy_(t)
        g.replay()
        torch.cuda.synchronize()
        adjust_check(logits, a, out.cpu().numpy())


# ---------------------------------------------------------------------------
# the operators together, as decode.BatchStep runs them
# ---------------------------------------------------------------------------
def make_step8(rng, T, B, ps, pages, window=0, seen=None, **kw):
    """A BatchStep over caches of 8 bits, of make_step's weights; `seen` receives
    (what, layer, input, output, q, codes and scales after it)."""
    base = make_step(rng, T, B, ps, pages, window)
    num, Hkv = base.k_pages[0].shape[:2]

    def watched(f, what, l):
        def g(x, out):
            f(x, out)
            if seen is not None:
                seen[what, l] = [x.clone(), out.clone(), step.q.clone()] + [
                    t.view(torch.uint8).clone() for t in (step.k_pages[l], step.v_pages[l], step.k_scales[l], step.v_scales[l])]
        return g
    lins = [tuple(watched(f, what, l) for f, what in zip(fs, ("qkv", "o", "gu", "down"))) for l, fs in enumerate(base.linears)]
    kp, vp = ([torch.zeros((num, Hkv, ps, 128), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)] for _ in range(2))
    ks, vs = ([torch.zeros((num, Hkv, ps // 16), dtype=torch.uint8, device=DEV).view(E8M0) for _ in range(2)] for _ in range(2))
    step = decode.BatchStep(SHAPE, lins, base.norms, base.final_norm, kp, vp, B, T, pages, DEV, lm_head=base.lm_head,
                            window=window, k_scales=ks, v_scales=vs, **kw)
    step.page_table.copy_(base.page_table)
    return step


@pytest.mark.parametrize("window", [0, 9])
def test_batch_step(window):
    """A prompt's chunk, a second chunk beside a decoding sequence, then decoding
    with padding rows: append and attention against the oracle from the stage's
    own inputs on the GPU, then penalties, biases and a mask, and the draw."""
    say("batch step8", window)
    rng = np.random.default_rng(170 + window)
    T, B, ps, pages, H, N = 12, 3, 16, 3, 20, 4
    seen = {}
    step = make_step8(rng, T, B, ps, pages, window, seen, history=H, biases=N, grammar=True)
    Hq, Hkv, V = SHAPE["heads"], SHAPE["kv_heads"], SHAPE["vocab"]
    cs = step.cos_sin.cpu().numpy()
    first = True
    for tokens, before in (([12, 0, 0], [0, 0, 0]), ([6, 5, 1], [12, 0, 0]), ([1, 1, 1], [18, 5, 1]),
                           ([1, 1, 1], [19, 6, 2])):
        set_rows(step, tokens, before, rng)
        step.u.copy_(dev(rng.random(T).astype(np.float32)))
        step.temperature.fill_(0.8)
        step.top_k.fill_(50)
        old = [[host(t) for t in ts] for ts in zip(step.k_pages, step.v_pages, step.k_scales, step.v_scales)]
        logits = step.run()
        if first:  # what changes nothing
            tok, prob = step.sample()
            assert torch.equal(step.adjusted.view(torch.int16), logits.view(torch.int16))
            first = False
        _, a = adjust_case(rng, T, V, H, N, True)
        for n, t in to_dev(a).items():
            getattr(step, n).copy_(t)
        tok, prob = step.sample()
        torch.cuda.synchronize()
        table, start, lens = (t.cpu().numpy() for t in (step.page_table, step.token_start, step.seq_len))
        mine = sum(tokens)
        for l in range(2):
            bt = Batch8.__new__(Batch8)
            bt.kc, bt.vc, bt.ks, bt.vs = old[l]
            bt.tokens, bt.table, bt.start, bt.lens, bt.T, bt.ps, bt.Hkv, bt.P = tokens, table, start, lens, T, ps, Hkv, len(bt.kc)
            qkv = seen["qkv", l][1].cpu().numpy()
            x, _, q, k, v, ks, vs = (t.cpu().numpy() for t in seen["o", l])
            check_append(rng, bt, qkv, *(w.cpu().numpy() for w in step.norms[l][2:]), step.cos_sin, Hq,
                         np.zeros((T, Hq, 128), np.float16), got=((k, ks), (v, vs)))
            bt.kc, bt.vc, bt.ks, bt.vs = k, v, ks, vs
            bt.values()
            check_rows(bt, Hq, q, np.concatenate([x.reshape(T, Hq, 128)[:mine], np.zeros((T - mine, Hq, 128), np.float16)]),
                       window, np.zeros((T, Hq, 128), np.float16))
        plain, adjusted = logits.cpu().numpy(), step.adjusted.cpu().numpy()
        adjust_check(plain, a, adjusted)
        for r in range(mine):
            want, p = OS.sample_row(adjusted[r], float(step.u[r]), temperature=float(np.float32(0.8)), top_k=50)
            assert int(tok[r]) == want and abs(float(prob[r]) - p) <= 2.0**-23 * p


def test_batch_step_in_a_graph():
    """A decoding loop that feeds each step's tokens into the next and into the
    histories, as graph replays and as eager calls: the same tokens, caches and
    logits; and penalties that forbid what was said are kept."""
    say("batch step8 graph")
    T, B, ps, pages, H = 4, 4, 16, 4, 16
    runs = []
    for graphed in (False, True):
        rng = np.random.default_rng(90)
        step = make_step8(rng, T, B, ps, pages, history=H)
        table = dev(rng.standard_normal((SHAPE["vocab"], SHAPE["hidden"])).astype(np.float32))
        one = torch.ones_like(step.seq_len)
        step.token_start.copy_(torch.arange(B + 1, device=DEV, dtype=torch.int32))
        step.temperature.copy_(torch.tensor([0.0, 0.7, 1.0, 1.3], device=DEV))
        step.top_k.fill_(20)
        step.presence.fill_(60000.0)  # no token twice

        def one_step():
            step.seq_len.add_(one)
            step.run()
            tok, _ = step.sample()
            step.history.scatter_(1, step.history_len.long()[:, None], tok[:, None])
            step.history_len.add_(one)
            torch.index_select(table, 0, tok, out=step.x0)
        state = [step.seq_len, step.x0, step.history, step.history_len] + [
            t.view(torch.uint8) for ts in (step.k_pages, step.v_pages, step.k_scales, step.v_scales) for t in ts]
        g, got = None, []
        uniform = rng.random((8, T)).astype(np.float32)
        step.x0.copy_(table[:T])
        for i in range(8):
            step.u.copy_(dev(uniform[i]))
            if graphed and i == 1:  # the first step, eager, warms up
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                saved = [t.clone() for t in state]
                with torch.cuda.graph(g):
                    one_step()
                for t, s in zip(state, saved):
                    t.copy_(s)
            if g is not None:
                g.replay()
            else:
                one_step()
            torch.cuda.synchronize()
            got.append([step.tokens.clone(), step.logits.view(torch.int16).clone(), step.adjusted.view(torch.int16).clone()])
        runs.append(got + [[t.clone() for t in state]])
        said = torch.stack([x[0] for x in got[:8]]).cpu().numpy()
        assert all(len(set(said[:, r])) == 8 for r in range(T))
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
