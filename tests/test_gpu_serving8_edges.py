"""Batched serving over caches of 8 bits and logits before sampling, at the
shapes where another path of a kernel begins.  Oracle, checks and tolerances are
test_gpu_serving8.py's, where nothing else is said.
"""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from oracle.compare import linear_check
from paper_2605_08755_amd import decode, laq
from test_gpu_serving import Batch, attention_check, dev, f16, say
from test_gpu_serving8 import (DEV, EPS, Batch8, adjust_case, adjust_check, attend, half_step, host, small,
                               to_dev)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
def append_shape(T, Hq, Hkv):
    """(rows of a window of the key and value waves, waves of a row's query
    heads): windows of 1, 2, 4, 8 or 16 rows whose waves are at most 8192, and as
    many query waves as 8192 leave a row, one per eight heads at most."""
    window = 1
    while window < 16 and -(-T // window) * 2 * Hkv > 8192:
        window *= 2
    return window, max(1, min((Hq + 7) // 8, 8192 // T))


def append_all(rng, bt, qkv, qw, kw, cs, Hq, qkv_dev=None, start=None, table=None):
    """An append on the batch's caches, everything that it writes against the
    oracle: query rows and those of no sequence, scales, values' codes, new keys
    (check_append's tolerance); and the key codes of all other positions, which
    are as they were or, where their scale grew, the oracle's (NaN for NaN only).
    start, table: what the call gets in the place of the batch's own."""
    k, v, ks, vs, own_table, own_start, lens = bt.device8()
    canary = f16(rng, (bt.T, Hq, 128))
    q = laq.paged_append_e4m3(dev(qkv) if qkv_dev is None else qkv_dev, None if qw is None else dev(qw),
                              None if kw is None else dev(kw), cs, k, v, ks, vs, own_table if table is None else table,
                              own_start if start is None else dev(start), lens, Hq, EPS, q_out=dev(canary))
    torch.cuda.synchronize()
    want_q, want = OS.paged_append_e4m3(qkv, qw, kw, cs.cpu().numpy(), ((bt.kc, bt.ks), (bt.vc, bt.vs)), bt.table, bt.start,
                                        bt.lens, Hq, EPS, canary)
    q = q.cpu().numpy()
    r = linear_check(q, want_q)
    assert r["ok"], r
    rest = np.setdiff1d(np.arange(len(q)), [r for r, _, _ in OS.rows(bt.start, bt.lens)])
    assert np.array_equal(q[rest].view(np.uint16), canary[rest].view(np.uint16))
    for name, codes, scales, (wcodes, wscales, exact) in zip("kv", (host(k), host(v)), (host(ks), host(vs)), want):
        assert np.array_equal(scales, wscales), name
        same = (codes == wcodes) | ((codes & 127) == 127) & ((wcodes & 127) == 127)
        new = ~np.isnan(exact)
        assert same[~new].all(), name
        if name == "v":
            assert same.all()
            continue
        x, got = exact[new.any(-1)], OS.e4m3_values()[codes[new.any(-1)]]  # [rows][128]
        pair = np.hypot(x[:, :64], x[:, 64:])
        slack = 2.0**-16 * np.concatenate([pair, pair], axis=-1)
        x = np.clip(x, -448, 448)
        assert (np.abs(got - x) <= half_step(np.abs(x) + slack) + slack).all()


def append_inputs(rng, bt, Hq, Hkv):
    """Rows of unlike magnitudes, norm weights."""
    width = (Hq + 2 * Hkv) * 128
    qkv = (rng.standard_normal((bt.T, width)) * np.exp(1.5 * rng.standard_normal((bt.T, 1)))).astype(np.float16)
    return (qkv,) + tuple((1 + 0.2 * rng.standard_normal(128)).astype(np.float16) for _ in range(2))


@pytest.mark.parametrize("window,q_waves,Hq,Hkv,ps,tokens,before,kw", [
    (8, 8, 64, 64, 16, [300], [5], {}),
    (8, 8, 64, 64, 32, [1, 2, 3, 0, 5, 40, 1, 1, 17, 225], [7, 15, 40, 0, 14, 3, 31, 16, 90, 11], {"pad": 3, "first": 2}),
    (8, 8, 64, 64, 16, [1] * 290, [7 * i % 48 for i in range(290)], {}),
    (16, 8, 64, 64, 16, [600], [9], {}),
    (16, 8, 64, 64, 64, [37, 1, 500, 80], [30, 63, 5, 0], {"slot_major": True}),
    (16, 8, 64, 64, 16, [1, 2, 0, 3, 20] * 23, [7, 15, 40, 30, 1] * 23, {"pad": 5, "first": 1}),
    (16, 3, 32, 32, 16, [2100], [3], {}),          # three waves for four groups of eight query heads
    (2, 1, 33, 1, 32, [2500, 1, 2499], [40, 17, 0], {}),  # one wave for five, the last of one head
    (1, 2, 24, 1, 16, [4095], [1], {}),            # two for three
])
def test_append_windows(window, q_waves, Hq, Hkv, ps, tokens, before, kw):
    """Windows of 8 and of 16 rows, with sequences that begin inside a block and
    several in one window; query waves that go on to further groups of heads."""
    say("append8 windows", window, q_waves, Hq, Hkv, ps, len(tokens), sum(tokens))
    rng = np.random.default_rng(sum(tokens) + Hq + ps)
    bt = Batch8(rng, tokens, before, ps, Hkv, garbage=None, spread=3, **kw)
    assert append_shape(bt.T, Hq, Hkv) == (window, q_waves)
    cs = decode.rope_table(int(bt.lens.max()) + 1, 1e6, DEV)
    append_all(rng, bt, *append_inputs(rng, bt, Hq, Hkv), cs, Hq)


@pytest.mark.parametrize("T,window", [(300, 8), (600, 16)])
def test_append_windows_of_places_that_are_not_there(T, window):
    """Missing pages and pages outside the cache, negative positions, positions
    past the rotation table and past the page table, among the rows of a window;
    row starts below 0 and past T."""
    say("append8 windows, bad places", T)
    rng = np.random.default_rng(T)
    Hq = Hkv = 64
    n = T // 6
    tokens, before = [n] * 5 + [T - 5 * n], [3, 30, 17, 0, 9, 100]
    bt = Batch8(rng, tokens, before, 16, Hkv, garbage=None)
    assert append_shape(T, Hq, Hkv)[0] == window
    bt.table[0, 1], bt.table[2, 2], bt.table[4, 0] = -1, bt.P, 2**31 - 1
    bt.lens[1] = n - 7  # the first seven at negative positions
    bt.lens[3] = -5     # all of them
    bt.lens[5] = bt.table.shape[1] * 16 + 20  # the last 20 past the page table
    inputs = append_inputs(rng, bt, Hq, Hkv)
    start = bt.start.copy()
    start[0], start[-1] = -50, T + 1000
    for positions in (400, 70):
        cs = decode.rope_table(positions, 1e6, DEV)
        append_all(rng, bt, *inputs, cs, Hq)
        append_all(rng, bt, *inputs, cs, Hq, start=start)


def test_append_query_rows_of_views():
    """Query rows where rows and page tables are views of wider arrays."""
    say("append8 views")
    rng = np.random.default_rng(2)
    Hq, Hkv = 6, 2
    bt = Batch8(rng, [5, 1, 18], [9, 40, 3], 16, Hkv, garbage=None)
    qkv, qw, kw = append_inputs(rng, bt, Hq, Hkv)
    wide = np.full((bt.T, qkv.shape[1] + 40), 9.0, dtype=np.float16)
    wide[:, 8:8 + qkv.shape[1]] = qkv
    table = torch.full((3, bt.table.shape[1] + 5), 77, dtype=torch.int32, device=DEV)
    table[:, 2:2 + bt.table.shape[1]] = dev(bt.table)
    append_all(rng, bt, qkv, qw, kw, decode.rope_table(64, 1e6, DEV), Hq, qkv_dev=dev(wide)[:, 8:8 + qkv.shape[1]],
               table=table[:, 2:2 + bt.table.shape[1]])


def test_append_keeps_key_codes():
    """Every key code before a block's new row, NaN among them, kept where the
    scale stays and rounded again where it grows; what belongs to others as it was."""
    say("append8 key codes")
    rng = np.random.default_rng(6)
    Hq, Hkv, ps = 2, 2, 16
    cs = torch.cat([torch.ones(600, 64), torch.zeros(600, 64)], dim=1).to(DEV).contiguous()  # no rotation
    for grow in (0, 1, 2, 7, 11, 22):
        bt = Batch8(rng, [1, 1, 3], [2, 15, 7], ps, Hkv, garbage=None)
        bt.kc = rng.permutation(np.resize(np.arange(256, dtype=np.uint8), bt.kc.size)).reshape(bt.kc.shape)
        bt.ks[:], bt.vs[:] = 112, 112
        qkv = f16(rng, (bt.T, (Hq + 2 * Hkv) * 128)).astype(np.float64)
        qkv = (np.clip(qkv, -4, 4) * 1.7 * 2.0**(grow - 15 + 6)).astype(np.float16)
        qkv[:, Hq * 128] = 1.75 * 2.0**(grow - 15 + 8)  # the largest key of head 0 fits scale 112 + grow
        append_all(rng, bt, qkv, None, None, cs, Hq)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_picked(bt, Hq, q, got, picked, window=0):
    """Some rows (row, sequence, position) of an attention against the definition in 64 bits."""
    R, few = Hq // bt.Hkv, small(bt, Hq)
    for r, b, pos in picked:
        t = np.arange(max(0, pos - window + 1) if window else 0, pos + 1)
        pages = bt.table[b, t // bt.ps]
        t, pages = t[(pages >= 0) & (pages < bt.P)], pages[(pages >= 0) & (pages < bt.P)]
        for g in range(bt.Hkv):
            K, V = (c[pages, g, t % bt.ps].astype(np.float64) for c in (bt.k, bt.v))
            x = q[r, R * g:R * (g + 1)].astype(np.float64)
            s = x @ K.T / 128**0.5
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            weight, reach = p @ np.abs(V), (np.abs(x) @ np.abs(K).T).max(1) / 128**0.5
            if few[b]:  # (2^-20 of the weights, with the output's own rounding)
                weight, reach = weight * (1 + 2.0**-7), reach + 2.0
            attention_check(got[r, R * g:R * (g + 1)], p @ V, weight, reach, len(t), not few[b])


SCALES = list(range(112, 135)) + [0, 111, 135, 255]


@pytest.mark.parametrize("n,Hq,Hkv", [(1, 2, 2), (20, 2, 2), (80, 64, 8)])
def test_attention_every_key_code_and_scale(n, Hq, Hkv):
    """A sequence for every scale, and those outside the range as its borders:
    position t holds code t (of odd heads 128 + t) in dimension t alone, and rows
    hold what makes each score a moderate number (as far as fp16 reaches), so that
    every code weighs its position's values.  By the kernel of 16 rows, and those
    of 128 and of 256 rows a block."""
    say("attention8 key codes", n, Hq, Hkv)
    rng = np.random.default_rng(n)
    tokens = [n] * len(SCALES)
    bt = Batch8(rng, tokens, [128] * len(SCALES), 16, Hkv)
    assert {1: bt.T * Hq <= 16 * Hkv * len(tokens), 20: 16 * Hkv * len(tokens) < bt.T * Hq < 512 * 256,
            80: bt.T * Hq >= 512 * 256}[n] and (n == 1 or n * (Hq // Hkv) > 16)
    code = np.arange(128)
    code[127] = 0  # (127 is NaN)
    bt.kc[bt.used[:, None].repeat(Hkv, 1)] = 0  # the rows' own keys are 0
    for i, s in enumerate(SCALES):
        for g in range(Hkv):
            for t in range(128):
                bt.kc[bt.table[i, t // 16], g, t % 16, t] = code[t] + 128 * (g & 1)
            bt.ks[bt.table[i, :8], g] = s
    bt.values()
    exponent = np.repeat([min(max(s, 112), 134) - 127 for s in SCALES], n)
    size = np.ldexp(np.maximum(OS.e4m3_values()[code], 2.0**-9), exponent[:, None])  # [T][128]
    wish = 2 * rng.standard_normal((bt.T, Hq, 128)) * 128**0.5 / size[:, None]
    q = np.clip(wish, -60000, 60000).astype(np.float16)
    got = attend(bt, q)
    again = attend(bt, q)
    assert np.array_equal(got.view(np.uint16), again.view(np.uint16))
    rows = list(OS.rows(bt.start, bt.lens))
    check_picked(bt, Hq, q, got, rows if n < 80 else [rows[n * i + j] for i in range(len(SCALES)) for j in (0, 37, n - 1)])


@pytest.mark.parametrize("tokens,before,Hq", [([1, 1], [60, 1500], 4), ([40], [90], 4), ([300, 1], [50, 700], 4),
                                              ([1] * 70, [40 + 9 * i for i in range(70)], 2)])
def test_attention_huge_scores_choose_a_value(tokens, before, Hq):
    """Scores from 2^20 on: where the largest is past all others by more than what
    32 bits can be off (136 x 2^-24 of the products' magnitudes, each) and 30, the
    output is the value of its position, e^-30 of the others apart."""
    say("huge scores8, values", tokens[:3])
    rng = np.random.default_rng(7 + sum(tokens))
    bt = Batch8(rng, tokens, before, 16, 2)
    bt.ks[:] = rng.choice([126, 131, 134], bt.ks.shape)
    bt.values()
    q = f16(rng, (bt.T, Hq, 128), 2000.0)
    got = attend(bt, q).astype(np.float64)
    clear = total = 0
    for r, b, pos in OS.rows(bt.start, bt.lens):
        t = np.arange(pos + 1)
        for h in range(Hq):
            K, V = (c[bt.table[b, t // 16], h // (Hq // 2), t % 16].astype(np.float64) for c in (bt.k, bt.v))
            x = q[r, h].astype(np.float64)
            s, off = K @ x / 128**0.5, 136 * 2.0**-24 * (np.abs(K) @ np.abs(x)) / 128**0.5
            top = int(np.argmax(s))
            rest = np.delete(s + off, top)
            total += 1
            if len(rest) and s[top] - off[top] - rest.max() <= 30:
                continue
            clear += 1
            tol = 2.0**-10 * np.abs(V[top]) + 2.0**-25 + len(t) * np.exp(-30.0) * np.abs(V).max()
            assert (np.abs(got[r, h] - V[top]) <= tol).all(), (r, h)
    assert clear >= 0.9 * total


@pytest.mark.parametrize("tokens,before,Hq,Hkv,window", [
    ([1] * 80, [37 * i % 800 for i in range(79)] + [3000], 8, 2, 100),
    ([1] * 80, [37 * i % 800 for i in range(79)] + [3000], 8, 2, 700),
    ([2, 0, 1] * 60, [100, 5, 1400] * 60, 4, 4, 333),
    ([5] * 40 + [300] + [5] * 30, [20] * 40 + [1500] + [100] * 30, 4, 2, 200),
    ([1] * 50 + [170, 0, 33] * 6, [600] * 50 + [1800, 9, 64] * 6, 8, 2, 900),
    ([40] * 66, [1100] * 66, 4, 1, 64),
])
def test_attention_of_many_sequences_within_a_window(tokens, before, Hq, Hkv, window):
    """More than 64 sequences, whose plan a kernel of its own makes, with windows:
    each tile's own positions are its ranges."""
    say("attention8 many, window", tokens[:3], len(tokens), window)
    rng = np.random.default_rng(len(tokens) + window)
    bt = Batch8(rng, tokens, before, 16, Hkv, pad=3)
    for b, p in enumerate(before):  # pages that no row sees were given back
        bt.table[b, :max(0, p - window + 1) // 16] = -1
    q, canary = f16(rng, (bt.T, Hq, 128), 1.5), f16(rng, (bt.T, Hq, 128))
    got = attend(bt, q, window, dev(canary))
    assert np.array_equal(got[-3:], canary[-3:])
    assert np.array_equal(got.view(np.uint16), attend(bt, q, window, dev(canary)).view(np.uint16))
    rows = list(OS.rows(bt.start, bt.lens))
    picked = rows if len(rows) <= 200 else [rows[i] for i in sorted(rng.choice(len(rows), 200, replace=False))]
    check_picked(bt, Hq, q, got, picked, window)


@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("tokens,before,Hq,Hkv", [
    ([1] * 60 + [1] * 4, [100] * 60 + [5000, 3001, 2500, 4000], 64, 8),
    ([2] * 50 + [1, 2, 2], [70] * 50 + [4000, 4100, 1500], 64, 8),
    ([1] * 90 + [1] * 3, [20 + i for i in range(90)] + [3000, 6000, 2222], 128, 8),
    ([1] * 40, [50 * i for i in range(40)], 56, 8),
])
def test_attention_rows_joined_in_turns(tokens, before, Hq, Hkv, codes):
    """Batches with more rows to join than blocks that run at once: a block joins
    one row after another.  Over both types of cache."""
    say("joined in turns", len(tokens), Hq, Hkv, codes)
    rng = np.random.default_rng(len(tokens) + Hq)
    R, T, B = Hq // Hkv, sum(tokens), len(tokens)
    split_tiles = min(-(-512 // Hkv), (T * R + B * 15) // 16) * Hkv  # as many as can be split
    assert 16 * split_tiles > 4096 and 2048 // (split_tiles + 1) < max(tokens) * R and T * R <= 16 * B
    bt = (Batch8 if codes else Batch)(rng, tokens, before, 16, Hkv)
    q, canary = f16(rng, (T, Hq, 128), 1.5), f16(rng, (T, Hq, 128))
    if codes:
        got = attend(bt, q, 0, dev(canary))
    else:
        got = laq.paged_attention(dev(q), *bt.device(), out=dev(canary))
        torch.cuda.synchronize()
        got = got.cpu().numpy()
    check_picked(bt, Hq, q, got, list(OS.rows(bt.start, bt.lens)))


@pytest.mark.parametrize("beside", [False, True])
def test_attention_of_few_rows_cuts_small_probabilities_off(beside):
    """Probabilities of a sequence of up to 16 query rows are cut off at 22 bits, or
    at 2^-32 of the largest where that is more.

    Every 32nd position has the score that all others are some 2^-10 to 2^-20 of, and
    values of 0.  The others' values are A and -A with one score for each sign, so
    that what is cut off adds up.  Scores are one product each (exact) times a
    constant in 32 bits, less a reference, and an exponential: four roundings of
    the exponent's size (2^-24 of it) and two of the result; sums of L positions in
    32 bits: L x 2^-24 of the magnitudes; the output's rounding 2^-11."""
    say("few rows8, small probabilities", beside)
    rng = np.random.default_rng(77)
    n, L = 48, 64
    tokens, before = [1] * n + [900] * beside, [L - 1] * n + [40] * beside  # (900: the kernel of chunks)
    bt = Batch8(rng, tokens, before, 16, 1)
    bt.kc[:], bt.vc[:] = 0, 0
    bt.ks[:], bt.vs[:] = 127, 134
    q = f16(rng, (bt.T, 1, 128))
    for b in range(n):
        sign = rng.permutation(np.resize([0, 1], L))
        for t in range(L):
            at = bt.table[b, t // 16], 0, t % 16
            bt.kc[at][0] = 0x40 if t % 32 == 0 else 0  # 2
            bt.kc[at][1] = 0x38 if t % 32 and sign[t] else 0  # 1
            bt.vc[at] = 0 if t % 32 == 0 else 0xFE if sign[t] else 0x7E  # 57344 or less
        q[b, 0] = 0
        q[b, 0, 0] = (10 + 10 * b / n) * np.log(2) * 128**0.5 / 2
        q[b, 0, 1] = rng.uniform(-0.2, 0.2)
    bt.values()
    got = attend(bt, q).astype(np.float64)
    for b in range(n):
        t = np.arange(L)
        K, V = (c[bt.table[b, t // 16], 0, t % 16].astype(np.float64) for c in (bt.k, bt.v))
        s = K @ q[b, 0].astype(np.float64) / 128**0.5
        p = np.exp(s - s.max())
        den, V = p.sum(), V[:, 0]
        ref = p @ V / den
        moved = 4 * 2.0**-24 * np.abs(s).max() + 2 * 2.0**-24 + 2 * L * 2.0**-24
        cut = (np.maximum(2.0**-21 * p, 2.0**-32) @ np.abs(V)) / den
        tol = 2.0**-11 * abs(ref) + 2 * moved * (p @ np.abs(V)) / den + cut + 2.0**-25
        assert (np.abs(got[b, 0] - ref) <= tol).all(), (b, float(np.abs(got[b, 0] - ref).max()), tol)


# ---------------------------------------------------------------------------
# logits before sampling
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("R,V,H,N,mask", [(1, 5, 3, 2, True), (3, 4001, 60, 5, True), (5, 8200, 0, 0, False),
                                          (300, 7001, 64, 4, True), (2, 70001, 17000, 300, True)])
def test_adjust_into_columns_beside_the_logits(R, V, H, N, mask):
    """Logits and out as columns of one array, either first, and as rows of
    unlike strides between each other: the bits of a call with arrays of their
    own, nothing beside out written."""
    say("adjust columns", R, V, H, N, mask)
    rng = np.random.default_rng(R + V)
    logits, a = adjust_case(rng, R, V, H, N, mask)
    d = to_dev(a)
    want = laq.adjust_logits(dev(logits), **d)
    torch.cuda.synchronize()
    adjust_check(logits, a, want.cpu().numpy())
    for gap in (0, 3, 8):
        for first in (True, False):
            both = torch.full((R, 2 * V + gap + 5), 7.0, dtype=torch.float16, device=DEV)
            x, y = both[:, :V], both[:, V + gap:2 * V + gap]
            if not first:
                x, y = y, x
            x.copy_(dev(logits))
            before = both.clone()
            got = laq.adjust_logits(x, **d, out=y)
            torch.cuda.synchronize()
            assert got.data_ptr() == y.data_ptr() and torch.equal(y.view(torch.int16), want.view(torch.int16))
            y.copy_(before[:, V + gap:2 * V + gap] if first else before[:, :V])
            assert torch.equal(both.view(torch.int16), before.view(torch.int16))
    # out's rows between the logits', whose stride is twice theirs: row i of out at V + i 2 V, of the logits at i 4 V
    flat = torch.full((4 * V * (R + 1),), 7.0, dtype=torch.float16, device=DEV)
    x, y = flat.as_strided((R, V), (4 * V, 1)), flat.as_strided((R, V), (2 * V, 1), V)
    x.copy_(dev(logits))
    laq.adjust_logits(x, **d, out=y)
    torch.cuda.synchronize()
    assert torch.equal(y.view(torch.int16), want.view(torch.int16)) and torch.equal(x.view(torch.int16), dev(logits).view(torch.int16))
    with pytest.raises(laq.LaqError):
        laq.adjust_logits(x, **d, out=flat.as_strided((R, V), (4 * V, 1), V - 1))
