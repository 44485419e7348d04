"""Batched serving operations on the GPU (paged append, paged attention,
sampling) against the float64 oracle (oracle/serving.py).

Tolerances, from the arithmetic:
  append     fp32 steps on fp16 inputs, one fp16 rounding: linear_check.
  attention  one fp16 rounding of the output (2^-11 of it), and relative to
             the weights' sum of |v|: scores are fp32 sums of 128 exact
             products (128 x 2^-24 of the sum of their magnitudes; eight more
             for the scale, the exponent's argument and the exponential), which
             move every weight and the denominator by that much; sums over L
             positions (L x 2^-24 in value sums and denominator); and where
             probabilities are rounded to fp16, 2^-11.
  sample     tokens equal; probabilities within fp32 rounding.
"""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from oracle.compare import linear_check
from paper_2605_08755_amd import decode, laq

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
EPS = 1e-6


def say(*a):
    print("[gpu-case]", *a, flush=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def f16(rng, shape, scale=1.0):
    return (rng.standard_normal(shape) * scale).astype(np.float16)


class Batch:
    """Sequences of the given new rows and earlier positions, their pages in
    random order; `spare` pages belong to nobody, and unused slots hold NaN."""

    def __init__(self, rng, tokens, before, ps, Hkv, pad=0, first=0, spare=2, extra_columns=0, slot_major=False,
                 garbage=np.nan):
        self.tokens, self.before, self.ps, self.Hkv = tokens, before, ps, Hkv
        self.lens = np.array([n + p for n, p in zip(tokens, before)], dtype=np.int32)
        self.start = (first + np.concatenate([[0], np.cumsum(tokens)])).astype(np.int32)
        self.T = int(self.start[-1]) + pad
        pages = [-(-int(n) // ps) for n in self.lens]
        self.P = sum(pages) + spare
        self.table = np.full((len(tokens), max(max(pages), 1) + extra_columns), -1, dtype=np.int32)
        order = rng.permutation(self.P).astype(np.int32)
        used = np.zeros((self.P, ps), dtype=bool)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = order[at:at + n]
            at += n
            for t in range(int(self.lens[b])):
                used[self.table[b, t // ps], t % ps] = True
        self.used = used
        self.slot_major = slot_major
        self.k, self.v = (f16(rng, (self.P, Hkv, ps, 128)) for _ in range(2))
        if garbage is not None:
            for c in (self.k, self.v):
                c[np.broadcast_to(~used[:, None], (self.P, Hkv, ps))] = garbage

    def cache(self, c):
        if self.slot_major:
            return dev(c.transpose(0, 2, 1, 3)).transpose(1, 2)
        return dev(c)

    def device(self):
        return (self.cache(self.k), self.cache(self.v), dev(self.table), dev(self.start), dev(self.lens))


def attention_check(out, ref, weight, reach, L, fp16_probs):
    out = out.astype(np.float64)
    assert np.isfinite(out).all()
    rel = 2 * (136 * 2.0**-24 * reach)[..., None] + 2 * L * 2.0**-24 + (2.0**-11 if fp16_probs else 0.0)
    tol = 2.0**-11 * np.abs(ref) + rel * weight * (1 + 2.0**-10) + 2.0**-25
    bad = np.abs(out - ref) > tol
    assert not bad.any(), (int(bad.sum()), float((np.abs(out - ref) / tol).max()), np.argwhere(bad)[:4].tolist())


def run_attention(rng, bt, Hq, window=0, q_scale=1.5, check=True):
    q = f16(rng, (bt.T, Hq, 128), q_scale)
    canary = f16(rng, (bt.T, Hq, 128))
    out = dev(canary)
    k, v, table, start, lens = bt.device()
    got = laq.paged_attention(dev(q), k, v, table, start, lens, window=window, out=out)
    torch.cuda.synchronize()
    got = got.cpu().numpy()
    if check:
        ref, weight, reach = OS.paged_attention(q, bt.k, bt.v, bt.table, bt.start, bt.lens, window, canary)
        fp16_probs = bt.T * (Hq // bt.Hkv) > 16 * len(bt.tokens)
        mine = np.zeros(bt.T, dtype=bool)
        mine[bt.start[0]:bt.start[-1]] = True
        attention_check(got[mine], ref[mine], weight[mine], reach[mine], int(bt.lens.max()), fp16_probs)
        assert np.array_equal(got[~mine], canary[~mine])  # rows of no sequence
    return q, got


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("Hq,Hkv,ps,tokens,before,kw", [
    (32, 8, 16, [1], [0], {}),
    (32, 8, 16, [1, 1, 1], [15, 16, 700], {}),
    (1, 1, 16, [5], [3], {}),
    (14, 2, 32, [3, 0, 17, 1], [31, 9, 0, 64], {"pad": 5}),
    (28, 4, 64, [66, 1], [0, 63], {"slot_major": True}),
    (40, 8, 16, [9, 40], [2, 0], {"first": 3, "pad": 2}),
    (64, 8, 256, [130], [200], {}),
    (3, 3, 16, [1] * 70, list(range(70)), {}),
    (8, 8, 16, [2100], [5], {}),
])
@pytest.mark.parametrize("norm", ["both", "q", "none"])
def test_append(Hq, Hkv, ps, tokens, before, kw, norm):
    say("append", Hq, Hkv, ps, len(tokens), sum(tokens), norm)
    if norm != "both" and sum(tokens) > 200:
        pytest.skip("norms covered by the smaller cases")
    rng = np.random.default_rng(sum(tokens) + Hq + ps)
    bt = Batch(rng, tokens, before, ps, Hkv, garbage=None, **kw)
    width = (Hq + 2 * Hkv) * 128
    wide = f16(rng, (bt.T, width + 24), 2.0)
    qw = (1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm != "none" else None
    kw_ = (1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm == "both" else None
    cs = decode.rope_table(int(bt.lens.max()) + 1, 1e6, DEV)
    k, v, table, start, lens = bt.device()
    canary = f16(rng, (bt.T, Hq, 128))
    q_out = dev(canary)
    qkv = dev(wide)[:, :width]  # strided rows
    got = laq.paged_append(qkv, None if qw is None else dev(qw), None if kw_ is None else dev(kw_), cs, k, v, table,
                           start, lens, Hq, EPS, q_out=q_out)
    torch.cuda.synchronize()
    assert got is q_out
    ref_q, ref_k, ref_v = OS.paged_append(wide[:, :width], qw, kw_, cs.cpu().numpy(), bt.k, bt.v, bt.table, bt.start,
                                          bt.lens, Hq, EPS, canary)
    q_h, k_h, v_h = got.cpu().numpy(), k.cpu().numpy(), v.cpu().numpy()
    for a, b in ((q_h, ref_q), (k_h, ref_k)):
        r = linear_check(a, b)
        assert r["ok"], r
    assert np.array_equal(v_h, ref_v.astype(np.float16))
    written = np.zeros((bt.P, ps), dtype=bool)
    for _, b, pos in OS.rows(bt.start, bt.lens):
        written[bt.table[b, pos // ps], pos % ps] = True
    keep = np.broadcast_to(~written[:, None], (bt.P, Hkv, ps))
    assert np.array_equal(k_h[keep], bt.k[keep]) and np.array_equal(v_h[keep], bt.v[keep])
    out_of_any = np.ones(bt.T, dtype=bool)
    out_of_any[bt.start[0]:bt.start[-1]] = False
    assert np.array_equal(q_h[out_of_any], canary[out_of_any])


def test_append_matches_single_token_call():
    """One row through laq.qk_norm_rope and through the paged call."""
    say("append vs qk_norm_rope")
    rng = np.random.default_rng(5)
    Hq, Hkv, pos, S = 32, 8, 37, 64
    qkv = dev(f16(rng, (1, (Hq + 2 * Hkv) * 128), 2.0))
    qw, kw = (dev((1 + 0.2 * rng.standard_normal(128)).astype(np.float16)) for _ in range(2))
    cs = decode.rope_table(S, 1e6, DEV)
    kc, vc = (torch.zeros((Hkv, S, 128), dtype=torch.float16, device=DEV) for _ in range(2))
    q1 = laq.qk_norm_rope(qkv, qw, kw, cs, pos, Hq, Hkv, EPS, kc, vc)
    kp, vp = (torch.zeros((4, Hkv, 16, 128), dtype=torch.float16, device=DEV) for _ in range(2))
    table = torch.tensor([[3, 1, 0, 2]], dtype=torch.int32, device=DEV)
    q2 = laq.paged_append(qkv, qw, kw, cs, kp, vp, table, torch.tensor([0, 1], dtype=torch.int32, device=DEV),
                          torch.tensor([pos + 1], dtype=torch.int32, device=DEV), Hq, EPS)
    torch.cuda.synchronize()
    for a, b in ((q2[0], q1), (kp[0, :, pos % 16], kc[:, pos])):  # one fp16 step apart at most
        a, b = a.float().cpu().numpy(), b.float().cpu().numpy()
        assert (np.abs(a - b) <= 2.0**-10 * np.abs(b) + 2.0**-24).all()
    assert torch.equal(vp[0, :, pos % 16], vc[:, pos])


def test_append_places_that_are_not_there():
    """Positions outside the rotation table or the page table, pages outside
    the cache: q zero or computed, nothing appended anywhere."""
    say("append bad places")
    rng = np.random.default_rng(11)
    Hq, Hkv, ps = 4, 2, 16
    P = 3
    k0 = f16(rng, (P, Hkv, ps, 128))
    table = np.array([[0, -1], [P, 1], [2, 2**31 - 1], [0, 1], [1, 1]], dtype=np.int32)
    # seq 0: position 16, page -1; 1: position 3, page P; 2: position 20, a huge page;
    # 3: position 32, past the page table; 4: two rows at positions -1 and 0 (page 1)
    lens = np.array([17, 4, 21, 33, 1], dtype=np.int32)
    start = np.array([0, 1, 2, 3, 4, 6], dtype=np.int32)
    qkv = f16(rng, (6, (Hq + 2 * Hkv) * 128))
    for S in (40, 17):  # with 17 rows of rotations, position 20 has none either
        cs = decode.rope_table(S, 1e6, DEV)
        k, v = dev(k0), dev(k0)
        q = laq.paged_append(dev(qkv), None, None, cs, k, v, dev(table), dev(start), dev(lens), Hq, EPS)
        torch.cuda.synchronize()
        ref = OS.paged_append(qkv, None, None, cs.cpu().numpy(), k0, k0, table, start, lens, Hq, EPS,
                              np.zeros((6, Hq, 128)))
        for a, b in zip((q, k, v), ref):
            r = linear_check(a.cpu().numpy(), b)
            assert r["ok"], r
        assert not q[3].any() and not q[4].any() and bool(q[2].any()) == (S == 40)
        assert np.array_equal(k.cpu().numpy()[1, :, 1:], k0[1, :, 1:]) and np.array_equal(k.cpu().numpy()[[0, 2]], k0[[0, 2]])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("Hq,Hkv,ps,tokens,before,window,kw", [
    # decoding: one row a sequence, lengths around steps, tiles and ranges
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
])
def test_attention(Hq, Hkv, ps, tokens, before, window, kw):
    say("attention", Hq, Hkv, ps, len(tokens), sum(tokens), max(before), window)
    rng = np.random.default_rng(sum(tokens) * 7 + sum(before) + Hq + window)
    bt = Batch(rng, tokens, before, ps, Hkv, **kw)
    if window:  # pages that no row sees were given back
        for b, p in enumerate(before):
            bt.table[b, :max(0, p - window + 1) // ps] = -1
    q, got = run_attention(rng, bt, Hq, window)
    # the same on every call
    k, v, table, start, lens = bt.device()
    again = laq.paged_attention(dev(q), k, v, table, start, lens, window=window)
    torch.cuda.synchronize()
    mine = slice(bt.start[0], bt.start[-1])
    assert np.array_equal(again.cpu().numpy()[mine].view(np.uint16), got[mine].view(np.uint16))


@pytest.mark.parametrize("tokens,before", [([1, 1], [2999, 20000]), ([40], [6000])])
def test_attention_long(tokens, before):
    """Many ranges per sequence, compared with torch in 64 bits."""
    say("attention long", tokens, before)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    Hq, Hkv, ps = 8, 2, 64
    lens = [n + p for n, p in zip(tokens, before)]
    width = -(-max(lens) // ps)
    P = len(tokens) * width
    k, v = (torch.randn((P, Hkv, ps, 128), generator=g, device=DEV).half() for _ in range(2))
    table = torch.randperm(P, generator=g, device=DEV).to(torch.int32).view(len(tokens), width)
    start = torch.tensor([0] + list(np.cumsum(tokens)), dtype=torch.int32, device=DEV)
    q = (1.5 * torch.randn((sum(tokens), Hq, 128), generator=g, device=DEV)).half()
    out = laq.paged_attention(q, k, v, table, start, torch.tensor(lens, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    R = Hq // Hkv
    for b, (n, L) in enumerate(zip(tokens, lens)):
        idx = table[b].long()
        for h in range(Hq):
            K = k[idx, h // R].reshape(-1, 128)[:L].double()
            V = v[idx, h // R].reshape(-1, 128)[:L].double()
            x = q[int(start[b]):int(start[b + 1]), h].double()
            s = x @ K.t().contiguous() / 128**0.5
            t = torch.arange(L, device=DEV)
            s.masked_fill_(t[None] > (L - n + torch.arange(n, device=DEV))[:, None], float("-inf"))
            p = torch.softmax(s, dim=-1)
            reach = ((x.abs() @ K.abs().t().contiguous()).amax(1) / 128**0.5).cpu().numpy()
            attention_check(out[int(start[b]):int(start[b + 1]), h].cpu().numpy(), (p @ V).cpu().numpy(),
                            (p @ V.abs()).cpu().numpy(), reach, L, sum(tokens) * R > 16 * len(tokens))


@pytest.mark.parametrize("Hq,tokens", [(2, [1, 1]), (2, [80, 3])])
def test_attention_large_scores(Hq, tokens):
    """Scores of several hundred, the largest first, last and in the middle:
    every other weight underflows, the running maximum jumps."""
    say("attention large scores", tokens)
    rng = np.random.default_rng(8)
    bt = Batch(rng, tokens, [300, 130], 16, 1)
    spikes = [0, 150, 299]
    for t in spikes:
        bt.k[bt.table[0, t // 16], 0, t % 16] = np.float16(30)
    run_attention(rng, bt, Hq, q_scale=8.0)


@pytest.mark.parametrize("tokens,before,window", [([1, 1], [100, 60], 0), ([4, 2], [90, 40], 48), ([70, 40], [90, 40], 0),
                                                  ([70, 40], [90, 40], 50)])
def test_attention_unseen_values(tokens, before, window):
    """Infinities and NaN among positions that a row does not see, keys and
    values, leave the row as it is; a row that sees one is not finite."""
    say("attention unseen", tokens, window)
    rng = np.random.default_rng(21)
    Hq, Hkv, ps = 4, 2, 16
    bt = Batch(rng, tokens, before, ps, Hkv)
    q, clean = run_attention(rng, bt, Hq, window)
    at = bt.lens[0] - 1 - (tokens[0] // 2 if tokens[0] > 1 else 0)  # a position that later rows alone see
    pg, sl = bt.table[0, at // ps], at % ps
    first = max(0, before[0] - window + 1) if window else 0
    for value in (np.inf, -np.inf, np.nan):
        k, v = bt.k.copy(), bt.v.copy()
        v[pg, 1, sl, ::3] = value
        k[pg, 0, sl, 5] = value
        if window and first > 0:  # and one before every window
            v[bt.table[0, (first - 1) // ps], 0, (first - 1) % ps] = value
        out = laq.paged_attention(dev(q), bt.cache(k), bt.cache(v), dev(bt.table), dev(bt.start), dev(bt.lens),
                                  window=window).cpu().numpy()
        for r, b, pos in OS.rows(bt.start, bt.lens):
            sees = b == 0 and pos >= at and (not window or pos - at < window)
            if not sees:
                assert np.array_equal(out[r].view(np.uint16), clean[r].view(np.uint16)), (r, pos, value)
            else:
                assert not np.isfinite(out[r, 2:, ::3]).any()
                assert np.array_equal(out[r, 2:, 1::3].view(np.uint16), clean[r, 2:, 1::3].view(np.uint16))


@pytest.mark.parametrize("tokens,before", [([1, 1], [700, 60]), ([70, 40], [90, 40]), ([2, 1], [30, 0])])
def test_attention_not_finite_inputs(tokens, before):
    """A NaN query head gives NaN and leaves the other heads and rows as they
    were; so does a NaN key for the rows and heads that see it."""
    say("attention not finite", tokens)
    rng = np.random.default_rng(22)
    Hq, Hkv, ps = 4, 2, 16
    bt = Batch(rng, tokens, before, ps, Hkv)
    q, clean = run_attention(rng, bt, Hq)
    bad = q.copy()
    bad[1, 2, 7] = np.nan
    out = laq.paged_attention(dev(bad), *bt.device()).cpu().numpy()
    assert np.isnan(out[1, 2]).all()
    out[1, 2] = clean[1, 2]
    assert np.array_equal(out.view(np.uint16), clean.view(np.uint16))
    bt.k[bt.table[0, 0], 1, 3, 9] = np.nan  # position 3 of the first sequence, heads 2 and 3
    out = laq.paged_attention(dev(q), *bt.device()).cpu().numpy()
    for r, b, pos in OS.rows(bt.start, bt.lens):
        if b == 0 and pos >= 3:
            assert np.isnan(out[r, 2:]).all()
            out[r, 2:] = clean[r, 2:]
    assert np.array_equal(out.view(np.uint16), clean.view(np.uint16))


@pytest.mark.parametrize("tokens", [[1, 1, 2], [40, 30, 9]])
def test_attention_rows_that_see_nothing(tokens):
    """No page of the sequence is there, the sequence has fewer positions than
    rows, its positions lie past the page table: zeros where nothing is seen."""
    say("attention nothing seen", tokens)
    rng = np.random.default_rng(33)
    bt = Batch(rng, tokens, [50, 20, 0], 16, 2)
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
    say("attention missing pages")
    rng = np.random.default_rng(4)
    for tokens, Hq in (([1, 1], 8), ([50, 20], 8)):
        bt = Batch(rng, tokens, [200, 90], 16, 2)
        bt.table[0, 3] = -1
        bt.table[0, 6] = bt.P + 5
        bt.table[1, 0] = -1
        run_attention(rng, bt, Hq)


@pytest.mark.parametrize("tokens,before,Hq,Hkv,ps,window", [
    ([255, 1, 0, 3], [1500, 300, 0, 1000], 1, 1, 16, 0),  # one row fewer than a block of 256 holds
    ([257, 2], [1800, 1023], 1, 1, 16, 0),                # and one more
    ([300, 5], [2300, 1100], 2, 1, 64, 1100),
    ([5] * 40 + [300] + [5] * 30, [20] * 40 + [1500] + [100] * 30, 4, 2, 16, 0),  # few joining blocks a tile
])
def test_attention_chunks_over_many_tiles(tokens, before, Hq, Hkv, ps, window):
    """Chunks of several blocks of rows over more positions than one set of
    page offsets covers (1024), pages missing around its ends, and infinities
    among the values that some rows of a block do not see."""
    say("attention many tiles", tokens[:4], Hq, Hkv, window)
    rng = np.random.default_rng(len(tokens) + Hq + ps)
    bt = Batch(rng, tokens, before, ps, Hkv)
    long = int(np.argmax(bt.lens))
    for at in (1000, 1023, 1024, 2040, 2064):
        if at < bt.lens[long]:
            bt.table[long, at // ps] = -1 if at != 1024 else bt.P
    q, clean = run_attention(rng, bt, Hq, window)
    at = int(bt.lens[long]) - 2  # the last two rows see it
    bt.v[bt.table[long, at // ps], 0, at % ps, ::5] = -np.inf
    out = laq.paged_attention(dev(q), *bt.device(), window=window).cpu().numpy()
    R = Hq // Hkv
    for r, b, pos in OS.rows(bt.start, bt.lens):
        if b == long and pos >= at:
            assert (out[r, :R, ::5] == -np.inf).all()
            out[r, :R, ::5] = clean[r, :R, ::5]
    assert np.array_equal(out.view(np.uint16), clean.view(np.uint16))


def test_attention_far_pages():
    """Pages past 2^31 elements of the cache; the other pages are never read."""
    say("attention far pages")
    rng = np.random.default_rng(6)
    Hq, Hkv, ps = 4, 2, 64
    P = 2**31 // (Hkv * ps * 128) + 40
    k, v = (torch.empty((P, Hkv, ps, 128), dtype=torch.float16, device=DEV) for _ in range(2))
    bt = Batch(rng, [1, 30], [200, 100], ps, Hkv)
    far = P - bt.P
    table = np.where(bt.table >= 0, bt.table + far, -1).astype(np.int32)
    k[far:], v[far:] = dev(bt.k), dev(bt.v)
    q = f16(rng, (bt.T, Hq, 128))
    out = laq.paged_attention(dev(q), k, v, dev(table), dev(bt.start), dev(bt.lens))
    ref = laq.paged_attention(dev(q), dev(bt.k), dev(bt.v), dev(bt.table), dev(bt.start), dev(bt.lens))
    qkv = dev(f16(rng, (bt.T, (Hq + 2 * Hkv) * 128)))
    cs = decode.rope_table(300, 1e6, DEV)
    k2, v2 = dev(bt.k), dev(bt.v)
    laq.paged_append(qkv, None, None, cs, k, v, dev(table), dev(bt.start), dev(bt.lens), Hq, EPS)
    laq.paged_append(qkv, None, None, cs, k2, v2, dev(bt.table), dev(bt.start), dev(bt.lens), Hq, EPS)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    for a, b in ((k, k2), (v, v2)):
        assert torch.equal(a[far:].view(torch.int16), b.view(torch.int16))


def test_attention_shared_pages_and_order():
    """Two sequences read the same pages; a sequence's result does not depend
    on the order of its pages in the cache."""
    say("attention shared pages")
    rng = np.random.default_rng(9)
    bt = Batch(rng, [1, 1], [400, 400], 16, 2)
    shared = bt.table.copy()
    shared[1] = shared[0]
    q = f16(rng, (1, 8, 128)).repeat(2, axis=0)
    k, v = bt.device()[:2]
    out = laq.paged_attention(dev(q), k, v, dev(shared), dev(bt.start), dev(bt.lens))
    assert torch.equal(out[0], out[1])
    perm = rng.permutation(bt.P)
    k2, v2 = dev(bt.k[np.argsort(perm)]), dev(bt.v[np.argsort(perm)])
    out2 = laq.paged_attention(dev(q), k2, v2, dev(perm[shared].astype(np.int32)), dev(bt.start), dev(bt.lens))
    assert torch.equal(out, out2)


def test_batch_in_a_graph():
    """Append and attention captured once; the replays follow the arrays that
    the host changes between them."""
    say("graph")
    rng = np.random.default_rng(14)
    Hq, Hkv, ps, B = 8, 2, 16, 3
    width = 40
    P = B * width
    k, v = (torch.zeros((P, Hkv, ps, 128), dtype=torch.float16, device=DEV) for _ in range(2))
    table = dev(rng.permutation(P).astype(np.int32).reshape(B, width))
    start, lens = dev(np.array([0, 1, 2, 3], dtype=np.int32)), dev(np.array([1, 1, 1], dtype=np.int32))
    cs = decode.rope_table(width * ps, 1e6, DEV)
    qkv = torch.zeros((B, (Hq + 2 * Hkv) * 128), dtype=torch.float16, device=DEV)
    q = torch.zeros((B, Hq, 128), dtype=torch.float16, device=DEV)
    out = torch.zeros_like(q)
    ws = torch.empty(laq.paged_attention_workspace_bytes(B, B, Hq, Hkv, width * ps), dtype=torch.uint8, device=DEV)

    def step(q, out, k, v):
        laq.paged_append(qkv, None, None, cs, k, v, table, start, lens, Hq, EPS, q_out=q)
        laq.paged_attention(q, k, v, table, start, lens, out=out, workspace=ws)
    step(q, out, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(q, out, k, v)
    k2, v2, q2, out2 = k.clone(), v.clone(), q.clone(), out.clone()
    for i in range(5):
        lens.copy_(dev(np.array([1 + i, 300 + 50 * i, 620 - i], dtype=np.int32)))
        qkv.copy_(dev(f16(rng, qkv.shape)))
        graph.replay()
        step(q2, out2, k2, v2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(q, q2) and torch.equal(k, k2), i


def test_batch_on_another_stream():
    say("another stream")
    rng = np.random.default_rng(15)
    bt = Batch(rng, [1, 30], [900, 300], 16, 2)
    q = dev(f16(rng, (bt.T, 8, 128)))
    args = bt.device()
    ref = laq.paged_attention(q, *args)
    logits = dev(f16(rng, (3, 5000), 3))
    u = torch.tensor([0.1, 0.5, 0.9], device=DEV)
    tok = laq.sample(logits, u)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = laq.paged_attention(q, *args)
        tok2 = laq.sample(logits, u)
    s.synchronize()
    assert torch.equal(out, ref)
    assert torch.equal(tok[0], tok2[0]) and torch.equal(tok[1], tok2[1])


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def sample_check(logits, u, **kw):
    arrays = {n: None if a is None else dev(np.asarray(a, dtype=np.int32 if n == "top_k" else np.float32))
              for n, a in kw.items()}
    x = logits if isinstance(logits, torch.Tensor) else dev(logits)
    u = np.asarray(u, dtype=np.float32)
    tok, prob = laq.sample(x, dev(u), **arrays)
    torch.cuda.synchronize()
    host = x.cpu().numpy()
    for r in range(host.shape[0]):
        want, p = OS.sample_row(host[r], u[r], **{n: a[r] for n, a in kw.items() if a is not None})
        assert int(tok[r]) == want, (r, int(tok[r]), want, float(prob[r]), p, {n: a[r] for n, a in kw.items()})
        assert abs(float(prob[r]) - p) <= 2.0**-23 * p + 1e-12, (r, float(prob[r]), p)
    return tok


SETTINGS = [
    {},
    {"temperature": 0.0},
    {"temperature": 0.7, "top_k": 1},
    {"temperature": 0.6, "top_k": 20, "top_p": 0.95},
    {"temperature": 1.3, "top_p": 0.5},
    {"temperature": 1.0, "top_p": 0.999},
    {"temperature": 1.0, "min_p": 0.05},
    {"temperature": 2.0, "top_k": 37, "min_p": 0.001},
    {"temperature": 0.9, "top_k": 100000, "top_p": 0.9, "min_p": 0.01},
    {"temperature": 0.05, "top_p": 0.3},
    {"temperature": 100.0, "top_k": 1000},
    {"temperature": 1.0, "top_p": 0.0, "min_p": 1.0},
    {"temperature": 1.0, "top_p": 1.0, "min_p": 0.0, "top_k": 0},
    {"temperature": 1.0, "min_p": 5.0},
]


@pytest.mark.parametrize("V", [1, 2, 63, 500, 8191, 8193, 32003, 50000, 81921, 151936, 170001])
def test_sample(V):
    """Every setting on rows of a vocabulary (register variants and the one that reads
    the row again), odd row starts included."""
    say("sample", V)
    rng = np.random.default_rng(V)
    settings = SETTINGS if V <= 50000 else SETTINGS[::2] + SETTINGS[3:4]
    n = len(settings)
    wide = (rng.standard_normal((n, V + 3)) * 3).astype(np.float16)
    wide[:, V // 2] += np.float16(6)
    x = dev(wide)[:, 1:V + 1]  # rows at odd offsets
    u = rng.random(n).astype(np.float32)
    kw = {k: [s.get(k, d) for s in settings] for k, d in
          (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))}
    sample_check(x, u, **kw)
    sample_check(x, u)  # no settings at all


def test_sample_draws():
    """u from 0 to 1 over a small row: every token in turn, and the borders."""
    say("sample draws")
    rng = np.random.default_rng(2)
    row = (rng.standard_normal(40) * 2).astype(np.float16)
    u = np.concatenate([np.linspace(0, 1, 201), [np.nextafter(np.float32(1), np.float32(0)), -1.0, np.nan, 7.0]])
    x = np.repeat(row[None], len(u), axis=0)
    tok = sample_check(x, u)
    assert len(set(tok.tolist())) > 20
    sample_check(x, u, top_k=[7] * len(u), top_p=[0.8] * len(u))
    sample_check(x, u, min_p=[0.1] * len(u))


def test_sample_equal_logits():
    """Equal logits: the order is the index, prefixes end inside a value."""
    say("sample equal logits")
    V = 3000
    x = np.zeros((8, V), dtype=np.float16)
    x[:, 1::2] = -0.0  # equal to 0
    u = np.array([0.0, 0.25, 0.5, 0.75, 0.999, 0.1, 0.3, 0.9], dtype=np.float32)
    tok = sample_check(x, u, temperature=[1.0] * 8)
    assert tok.tolist()[:4] == [0, 750, 1500, 2250]
    sample_check(x, u, top_k=[1, 2, 10, 1500, 2999, 3000, 3001, 0])
    tok = sample_check(x, u, top_p=[0.5] * 8)
    assert max(tok.tolist()) < 1500
    sample_check(x, u, temperature=[0.0] * 8)
    rng = np.random.default_rng(3)
    few = rng.integers(-3, 3, (8, 20000)).astype(np.float16)  # six values
    sample_check(few, u, top_k=[5, 100, 4000, 0, 19999, 7, 0, 12], top_p=[0.9, 1, 0.5, 0.7, 1, 0.1, 0.999, 1])


def test_sample_repeated_values():
    """Values that occur 65536 times and more: alone, beside the value that
    shares their word of the histogram, among NaN, as both zeros."""
    say("sample repeated values")
    V = 140001
    rng = np.random.default_rng(12)
    x = (rng.standard_normal((8, V)) * 2).astype(np.float16)
    # the sortable numbers of a and b differ by 2^15: one word counts both
    a = np.float16(1.5)
    b = np.array([(int(a.view(np.uint16)) | 0x8000) ^ 0x7FFF], dtype=np.uint16).view(np.float16)[0]
    assert b < 0
    x[0] = a
    x[1, :70000], x[1, 70000:] = a, b
    x[2, ::2], x[2, 1::2] = b, a
    x[3, :66000] = b
    x[4, :65536] = a
    x[5, :70000] = np.nan
    x[6, ::2], x[6, 1::2] = 0.0, -0.0
    x[7, :65535] = a
    u = np.array([0.0, 0.3, 0.999, 0.5, 0.7, 0.2, 0.9999, 0.45], dtype=np.float32)
    for kw in ({}, {"top_k": [70001, 70001, 100000, 65536, 0, 5, 139999, 1]}, {"top_p": [0.6] * 8},
               {"temperature": [0.3] * 8, "min_p": [0.01] * 8}):
        sample_check(x, u, **kw)


def test_sample_masked_rows():
    """-inf, NaN and +inf among the logits, rows with one token or none left."""
    say("sample masked")
    rng = np.random.default_rng(4)
    V = 9000
    x = (rng.standard_normal((10, V)) * 2).astype(np.float16)
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = -np.inf
    x[2, 4321] = -65504
    x[3, rng.random(V) < 0.99] = -np.inf
    x[4, ::2] = np.nan
    x[5, [7, 8000, 8999]] = np.inf
    x[6] = np.float16(-65504)
    x[7] = np.float16(65504)
    x[8, :-1] = -np.inf
    x[9, rng.random(V) < 0.5] = -np.inf
    u = rng.random(10).astype(np.float32)
    for kw in ({}, {"top_k": [3] * 10}, {"top_p": [0.9] * 10}, {"min_p": [0.2] * 10}, {"temperature": [0.0] * 10},
               {"temperature": [1e-4] * 10}, {"temperature": [np.nan] * 10}, {"temperature": [1e30] * 10},
               {"top_k": [8999] * 10, "top_p": [np.nan] * 10, "min_p": [np.nan] * 10}):
        tok = sample_check(x, u, **kw)
        assert tok.tolist()[:3] == [-1, -1, 4321] and int(tok[5]) in (7, 8000, 8999)


def test_sample_distribution():
    """Evenly spread u give each token its share of the draws to one draw."""
    say("sample distribution")
    rng = np.random.default_rng(6)
    V, n = 30, 4096
    row = (rng.standard_normal(V) * 1.5).astype(np.float16)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tok, prob = laq.sample(dev(np.repeat(row[None], n, axis=0)), dev(u), top_p=dev(np.full(n, 0.9, dtype=np.float32)))
    tok, prob = tok.cpu().numpy(), prob.cpu().numpy()
    for t in set(tok.tolist()):
        assert abs((tok == t).sum() - prob[tok == t][0] * n) <= 1.0


# ---------------------------------------------------------------------------
# the operators together, as decode.BatchStep runs them
# ---------------------------------------------------------------------------
SHAPE = {"layers": 2, "hidden": 256, "heads": 8, "kv_heads": 2, "mlp": 384, "eps": EPS, "rope_theta": 1e6,
         "vocab": 1000}


def make_step(rng, T, B, ps, pages, window, seen=None):
    """A BatchStep of quantized linears; `seen` receives (what, layer, input,
    q, output) of the attention-side linears as they are called."""
    D, Hq, Hkv, I = SHAPE["hidden"], SHAPE["heads"], SHAPE["kv_heads"], SHAPE["mlp"]

    def linear(N, K, what, l):
        p = laq.quantize_w3g128(dev(f16(rng, (N, K), 0.05)))

        def f(x, out):
            laq.linear(x, *p, 3, out=out)
            if seen is not None:
                seen.append((what, l, x.clone(), out.clone(), step.q.clone(), step.k_pages[l].clone(),
                             step.v_pages[l].clone()))
        return f
    vec = lambda n: dev((1 + 0.1 * rng.standard_normal(n)).astype(np.float16))  # noqa: E731
    lins = [(linear((Hq + 2 * Hkv) * 128, D, "qkv", l), linear(D, Hq * 128, "o", l), linear(2 * I, D, "gu", l),
             linear(D, I, "down", l)) for l in range(2)]
    norms = [(vec(D), vec(D), vec(128), vec(128)) for _ in range(2)]
    num = B * pages + 1
    kp, vp = ([torch.zeros((num, Hkv, ps, 128), dtype=torch.float16, device=DEV) for _ in range(2)] for _ in range(2))
    head = laq.quantize_w3g128(dev(f16(rng, (SHAPE["vocab"], D), 0.2)))
    step = decode.BatchStep(SHAPE, lins, norms, vec(D), kp, vp, B, T, pages, DEV,
                            lm_head=lambda x, out: laq.linear(x, *head, 3, out=out), window=window)
    step.page_table.copy_(dev(rng.permutation(num)[:B * pages].astype(np.int32).reshape(B, pages)))
    return step


def set_rows(step, tokens, before, rng):
    step.token_start.copy_(dev(np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32)))
    step.seq_len.copy_(dev((np.array(tokens) + np.array(before)).astype(np.int32)))
    step.x0.copy_(dev(rng.standard_normal(tuple(step.x0.shape)).astype(np.float32)))


@pytest.mark.parametrize("window", [0, 9])
def test_batch_step(window):
    """A prompt's chunk, a second chunk beside a decoding sequence, then
    decoding with padding rows: every stage against the oracle, from the stage's
    own inputs on the GPU."""
    say("batch step", window)
    rng = np.random.default_rng(70 + window)
    T, B, ps, pages = 12, 3, 16, 3
    seen = []
    step = make_step(rng, T, B, ps, pages, window, seen)
    Hq, Hkv = SHAPE["heads"], SHAPE["kv_heads"]
    cs = step.cos_sin.cpu().numpy()
    for tokens, before in (([12, 0, 0], [0, 0, 0]), ([6, 5, 1], [12, 0, 0]), ([1, 1, 1], [18, 5, 1]),
                           ([1, 1, 1], [19, 6, 2])):
        set_rows(step, tokens, before, rng)
        step.u.copy_(dev(rng.random(T).astype(np.float32)))
        step.temperature.fill_(0.8)
        step.top_k.fill_(50)
        step.top_p.fill_(0.9)
        del seen[:]
        old = [(k.cpu().numpy(), v.cpu().numpy()) for k, v in zip(step.k_pages, step.v_pages)]
        logits = step.run()
        tok, prob = step.sample()
        torch.cuda.synchronize()
        table, start, lens = (t.cpu().numpy() for t in (step.page_table, step.token_start, step.seq_len))
        mine = sum(tokens)
        for l in range(2):
            got = {e[0]: [x.cpu().numpy() for x in e[2:]] for e in seen if e[1] == l}
            qkv = got["qkv"][1]
            rq, rk, rv = OS.paged_append(qkv, step.norms[l][2].cpu().numpy(), step.norms[l][3].cpu().numpy(), cs,
                                         *old[l], table, start, lens, Hq, EPS, np.zeros((T, Hq, 128)))
            x, _, q, k, v = got["o"]
            for a, b in ((q[:mine], rq[:mine]), (k, rk)):
                r = linear_check(a, b)
                assert r["ok"], r
            assert np.array_equal(v, rv.astype(np.float16))
            ref, weight, reach = OS.paged_attention(q, k, v, table, start, lens, window, np.zeros((T, Hq, 128)))
            attention_check(x.reshape(T, Hq, 128)[:mine], ref[:mine], weight[:mine], reach[:mine], int(lens.max()),
                            T * (Hq // Hkv) > 16 * B)
        host = logits.cpu().numpy()
        for r in range(mine):
            want, p = OS.sample_row(host[r], float(step.u[r]), temperature=float(np.float32(0.8)), top_k=50,
                                    top_p=float(np.float32(0.9)))
            assert int(tok[r]) == want and abs(float(prob[r]) - p) <= 2.0**-23 * p


def test_batch_step_in_a_graph():
    """A decoding loop that feeds each step's tokens into the next, as graph
    replays and as eager calls: the same tokens, caches and logits."""
    say("batch step graph")
    T, B, ps, pages = 4, 4, 16, 4
    runs = []
    for graphed in (False, True):
        rng = np.random.default_rng(90)
        step = make_step(rng, T, B, ps, pages, 0)
        table = dev(rng.standard_normal((SHAPE["vocab"], SHAPE["hidden"])).astype(np.float32))
        one = torch.ones_like(step.seq_len)
        step.token_start.copy_(torch.arange(B + 1, device=DEV, dtype=torch.int32))
        step.temperature.copy_(torch.tensor([0.0, 0.7, 1.0, 1.3], device=DEV))
        step.top_k.fill_(20)

        def one_step():
            step.seq_len.add_(one)
            step.run()
            tok, _ = step.sample()
            torch.index_select(table, 0, tok, out=step.x0)
        g = None
        got = []
        uniform = rng.random((8, T)).astype(np.float32)
        step.x0.copy_(table[:T])
        for i in range(8):
            step.u.copy_(dev(uniform[i]))
            if graphed and i == 1:  # the first step, eager, warms up
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                saved = step.seq_len.clone(), step.x0.clone()
                with torch.cuda.graph(g):
                    one_step()
                step.seq_len.copy_(saved[0])
                step.x0.copy_(saved[1])
            if g is not None:
                g.replay()
            else:
                one_step()
            torch.cuda.synchronize()
            got.append((step.tokens.clone(), step.logits.clone()))
        runs.append((got, [k.clone() for k in step.k_pages]))
    for (a, la), (b, lb) in zip(runs[0][0], runs[1][0]):
        assert torch.equal(a, b) and torch.equal(la.view(torch.int16), lb.view(torch.int16))
    for a, b in zip(runs[0][1], runs[1][1]):
        assert torch.equal(a, b)
