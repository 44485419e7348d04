"""Batched serving on the GPU where its arithmetic is at its edges, against the
float64 oracle (oracle/serving.py)."""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from oracle.compare import linear_check
from paper_2605_08755_amd import decode, laq
from test_gpu_serving import Batch, attention_check, dev, f16, sample_check, say
from test_gpu_serving import test_attention_not_finite_inputs as not_finite_inputs
from test_gpu_serving import test_attention_rows_that_see_nothing as rows_that_see_nothing
from test_gpu_serving import test_attention_unseen_values as unseen_values

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def attend(q, bt, window=0):
    out = laq.paged_attention(dev(q), *bt.device(), window=window)
    torch.cuda.synchronize()
    return out.cpu().numpy()


def rows_of(bt, sequences):
    return [r for r, b, _ in OS.rows(bt.start, bt.lens) if b in sequences]


@pytest.mark.parametrize("tokens,before,Hq,Hkv,kw", [
    ([40, 1], [900, 50], 1, 1, {}),
    ([1, 1, 150, 1, 2], [33, 60, 20, 47, 40], 8, 2, {}),   # decoding rows beside a chunk
    ([70, 1, 1], [0, 47, 61], 5, 1, {}),
    ([1, 1], [50, 61], 8, 2, {"pad": 60}),                 # decoding rows of a batch with padding
    ([1], [53], 4, 1, {"pad": 30, "first": 9}),
    ([4], [44], 4, 1, {"pad": 1}),                         # 16 query rows
    ([100, 1, 4], [300, 700, 640], 4, 1, {}),              # split over ranges of positions
])
def test_attention_of_few_rows_keeps_32_bits(tokens, before, Hq, Hkv, kw):
    """Sequences of up to 16 query rows a key/value head, whatever stands
    beside them: the probabilities are not rounded to 16 bits.

    Scores are small sums of four products and values are +1 and -1, as many of
    the one as of the other, so that outputs are near 0 and their own fp16
    rounding is small.  The bound, relative to the weights' sum of |v| = 1:
    scores are fp32 sums (their errors as in tests/test_gpu_serving.py, 136 x
    2^-24 of the sum of magnitudes, in a weight and in the denominator), L x
    2^-24 in the value sums and in the denominator, and the rounding of the
    output, 2^-11 of it.  A rounding of each probability to 16 bits would be
    2^-11 of it."""
    say("few rows", tokens, Hq, kw)
    rng = np.random.default_rng(sum(tokens) + sum(before) + Hq)
    bt = Batch(rng, tokens, before, 16, Hkv, **kw)
    for b, n in enumerate(bt.lens):
        for g in range(Hkv):
            signs = np.array([rng.permutation(np.resize([1.0, -1.0], n)) for _ in range(128)])
            for t in range(n):
                bt.v[bt.table[b, t // 16], g, t % 16] = signs[:, t]
    q = np.zeros((bt.T, Hq, 128), dtype=np.float16)
    q[..., 5::32] = f16(rng, (bt.T, Hq, 4), 0.5)
    got = attend(q, bt).astype(np.float64)
    ref, weight, reach = OS.paged_attention(q, bt.k, bt.v, bt.table, bt.start, bt.lens, 0, np.zeros_like(got))
    mine = rows_of(bt, [b for b, n in enumerate(tokens) if n * (Hq // Hkv) <= 16])
    assert len(mine) >= 1 and np.allclose(weight[mine], 1)
    seen = {r: pos + 1 for r, _, pos in OS.rows(bt.start, bt.lens)}
    L = np.array([seen[r] for r in mine])[:, None, None]
    tol = 2.0**-11 * np.abs(ref[mine]) + 2 * 136 * 2.0**-24 * reach[mine][..., None] + 2 * L * 2.0**-24 + 2.0**-25
    err = np.abs(got[mine] - ref[mine])
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("tokens,before", [([40], [90]), ([1, 2], [300, 70]), ([300, 1], [50, 700]), ([20], [5000]),
                                           ([200], [3000])])
@pytest.mark.parametrize("size", [400.0, 4000.0, 10000.0, 20000.0])
def test_attention_huge_scores(tokens, before, size):
    """Finite queries and keys whose scores pass 2^24, where 32 bits no longer
    hold whole numbers: the largest score takes all, and equal keys share it.

    A row is compared where the next lower score is further from the largest
    than both can be off (136 x 2^-24 of the sum of magnitudes each) plus 50,
    e^-50 being nothing beside one fp16 step.  Weights of equal scores are equal,
    so a row's output is the mean of at most three values: two roundings of
    2^-11 and sums of a few terms."""
    say("huge scores", tokens, size)
    rng = np.random.default_rng(int(size) + sum(tokens))
    Hq, Hkv, ps = 4, 2, 16
    bt = Batch(rng, tokens, before, ps, Hkv)
    grow = lambda a: np.clip(a.astype(np.float32) * size, -65504, 65504).astype(np.float16)  # noqa: E731
    bt.k = np.where(np.isnan(bt.k), bt.k, grow(np.nan_to_num(bt.k)))
    at = lambda b, t: (bt.table[b, t // ps], slice(None), t % ps)  # noqa: E731
    for b, n in enumerate(bt.lens):  # equal keys, near and far
        for t, s in ((1, 0), (n // 2, 0), (n - 1 - tokens[b], 7)):
            bt.k[at(b, t)] = bt.k[at(b, s)]
    q = grow(f16(rng, (bt.T, Hq, 128)))
    got = attend(q, bt).astype(np.float64)
    assert np.isfinite(got[rows_of(bt, range(len(tokens)))]).all()
    compared = 0
    for r, b, pos in OS.rows(bt.start, bt.lens):
        t = np.arange(pos + 1)
        for h in range(Hq):
            K, V = (c[bt.table[b, t // ps], h // 2, t % ps].astype(np.float64) for c in (bt.k, bt.v))
            x = q[r, h].astype(np.float64)
            s = K @ x / 128**0.5
            reach = (np.abs(K) @ np.abs(x)).max() / 128**0.5
            top = s >= s.max() - 1e-9 * reach  # the same products, whatever their order
            rest = s[~top].max() if (~top).any() else -np.inf
            if s.max() - rest < 2 * 136 * 2.0**-24 * reach + 50 or top.sum() > 3:
                continue
            compared += 1
            want, weight = V[top].mean(0), np.abs(V[top]).mean(0)
            assert (np.abs(got[r, h] - want) <= 2.0**-11 * np.abs(want) + (2.0**-11 + 2.0**-20) * weight + 2.0**-25).all()
    assert compared > sum(tokens)


@pytest.mark.parametrize("tokens,before", [([40], [90]), ([300, 1], [50, 700]), ([30], [4000]), ([1, 1], [60, 1500])])
def test_attention_huge_scores_near_each_other(tokens, before):
    """Scores from 2^20 to 2^37 of which a row sees some that lie a few steps of
    32 bits apart, growing or in any order.  All values are 1, so that outputs
    are 1 whatever the weights: each probability's rounding is 2^-11 of it, the
    output's 2^-11, and sums over L positions 2 L x 2^-24."""
    say("huge scores near each other", tokens)
    rng = np.random.default_rng(sum(tokens) + sum(before))
    bt = Batch(rng, tokens, before, 16, 1)
    L = int(bt.lens.max())
    bt.v = np.where(np.isnan(bt.v), bt.v, np.float16(1))
    for e in range(20, 38):
        for order in ("growing", "any"):
            a = np.float16(2.0**((e - 6) / 2))  # 64 products of a x a: about 2^e
            q = np.zeros((bt.T, 2, 128), dtype=np.float16)
            q[..., :64], q[:, 0, 64], q[:, 1, 65] = a, 2.0**max(e - 24, 0), 2.0**max(e - 24, 0)
            k = np.zeros((bt.P, 1, 16, 128), dtype=np.float16)
            k[..., :64] = a
            for b, n in enumerate(bt.lens):
                steps = rng.integers(-64, 64, (n, 2)).astype(np.float16)
                if order == "growing":
                    steps.sort(axis=0)
                for t in range(n):
                    k[bt.table[b, t // 16], 0, t % 16, 64:66] = steps[t]
            k[~np.broadcast_to(bt.used[:, None], k.shape[:3])] = np.nan
            out = laq.paged_attention(dev(q), bt.cache(k), *bt.device()[1:])
            torch.cuda.synchronize()
            got = out.cpu().numpy()[rows_of(bt, range(len(tokens)))].astype(np.float64)
            assert (np.abs(got - 1) <= 2.0**-11 + 2.0**-11 + 2 * L * 2.0**-24).all(), (e, order, got.min(), got.max())


# ---------------------------------------------------------------------------
# many sequences
# ---------------------------------------------------------------------------
def many(rng, B, T, Hq, Hkv, ps=16):
    """T rows spread over B sequences (most waiting where T < B), pages of one
    row's sequences only: (table, start, lens) and arrays of the caches."""
    owner = np.sort(rng.integers(0, B, T))
    start = np.concatenate([[0], np.cumsum(np.bincount(owner, minlength=B))]).astype(np.int32)
    tokens = np.diff(start)
    lens = (tokens + rng.integers(0, 3 * ps - tokens.max(), B)).astype(np.int32)
    width = 3
    pages = np.where(tokens > 0, -(-lens // ps), 0)
    table = np.full((B, width), -1, dtype=np.int32)
    order = rng.permutation(int(pages.sum())).astype(np.int32)
    column = np.arange(width) < pages[:, None]
    table[column] = order
    k, v = (f16(rng, (len(order), Hkv, ps, 128)) for _ in range(2))
    return table, start, lens, k, v


@pytest.mark.parametrize("B,T", [(63, 40), (64, 200), (65, 65), (129, 500), (4095, 1000), (4097, 3000), (70000, 900),
                                 (1 << 20, 300)])
def test_append_many_sequences(B, T):
    """Rows of sequences anywhere among many, most of which wait."""
    say("append many", B, T)
    rng = np.random.default_rng(B + T)
    Hq, Hkv = 2, 1
    table, start, lens, k, v = many(rng, B, T, Hq, Hkv)
    qkv = f16(rng, (T, (Hq + 2 * Hkv) * 128))
    cs = decode.rope_table(64, 1e6, DEV)
    kd, vd = dev(k), dev(v)
    q = laq.paged_append(dev(qkv), None, None, cs, kd, vd, dev(table), dev(start), dev(lens), Hq, 1e-6)
    torch.cuda.synchronize()
    ref = OS.paged_append(qkv, None, None, cs.cpu().numpy(), k, v, table, start, lens, Hq, 1e-6, np.zeros((T, Hq, 128)))
    for a, b in zip((q, kd, vd), ref):
        r = linear_check(a.cpu().numpy(), b)
        assert r["ok"], r


def check(got, q, bt_arrays, window, fp16_probs):
    table, start, lens, k, v = bt_arrays
    ref, weight, reach = OS.paged_attention(q, k, v, table, start, lens, window, np.zeros(q.shape))
    attention_check(got, ref, weight, reach, int(lens.max()), fp16_probs)


@pytest.mark.parametrize("B,T,Hq,window", [(64, 60, 4, 0), (65, 65, 4, 0), (129, 600, 4, 0), (129, 600, 2, 9),
                                           (200, 3000, 2, 0), (4096, 700, 2, 0), (4097, 2000, 1, 0),
                                           (70000, 900, 2, 20), (1 << 20, 300, 2, 0)])
def test_attention_many_sequences(B, T, Hq, window):
    """Rows of sequences anywhere among many, most of which wait."""
    say("attention many", B, T, Hq, window)
    rng = np.random.default_rng(B + T + Hq)
    table, start, lens, k, v = many(rng, B, T, Hq, 1)
    q = f16(rng, (T, Hq, 128))
    out = laq.paged_attention(dev(q), dev(k), dev(v), dev(table), dev(start), dev(lens), window=window)
    torch.cuda.synchronize()
    check(out.cpu().numpy(), q, (table, start, lens, k, v), window, T * Hq > 16 * B)


@pytest.mark.parametrize("tokens,Hq,Hkv", [
    ([1] * 200, 4, 2),
    ([1] * 70 + [200] + [0] * 60 + [90, 3], 8, 1),        # chunks in the second and third group
    ([2] * 64 + [0] * 64 + [33, 1] * 32 + [140], 8, 2),
])
def test_attention_many_sequences_split(tokens, Hq, Hkv):
    """Long sequences, split over ranges, in every group of a batch."""
    say("attention many split", len(tokens), sum(tokens))
    rng = np.random.default_rng(len(tokens))
    before = [int(x) for x in rng.integers(0, 60, len(tokens))]
    for b in range(5, len(tokens), 61):
        before[b] = 1500 + b
    bt = Batch(rng, tokens, before, 16, Hkv)
    q = f16(rng, (bt.T, Hq, 128))
    got = attend(q, bt)
    check(got, q, (bt.table, bt.start, bt.lens, bt.k, bt.v), 0, bt.T * (Hq // Hkv) > 16 * len(tokens))
    again = attend(q, bt)
    assert np.array_equal(got.view(np.uint16), again.view(np.uint16))


def test_attention_many_sequences_in_a_graph():
    """The plan of a batch of more than 64 sequences follows the arrays that the
    host changes between replays; what the workspace held before does not matter."""
    say("attention many graph")
    rng = np.random.default_rng(41)
    Hq, Hkv, B, width = 4, 2, 100, 60
    k, v = (dev(f16(rng, (B * width, Hkv, 16, 128))) for _ in range(2))
    table = dev(rng.permutation(B * width).astype(np.int32).reshape(B, width))
    start = dev(np.arange(B + 1, dtype=np.int32))
    lens = torch.ones((B,), dtype=torch.int32, device=DEV)
    q = torch.zeros((B, Hq, 128), dtype=torch.float16, device=DEV)
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    nbytes = laq.paged_attention_workspace_bytes(B, B, Hq, Hkv, width * 16)
    ws, ws2 = (torch.full((nbytes,), x, dtype=torch.uint8, device=DEV) for x in (255, 0))
    laq.paged_attention(q, k, v, table, start, lens, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        laq.paged_attention(q, k, v, table, start, lens, out=out, workspace=ws)
    for i in range(4):
        new = rng.integers(1, 20 + 300 * i, B).astype(np.int32).clip(max=width * 16)
        lens.copy_(dev(new))
        first = np.sort(rng.integers(0, B, B - 1)) if i % 2 else np.arange(1, B)
        start.copy_(dev(np.concatenate([[0], first, [B]]).astype(np.int32)))
        q.copy_(dev(f16(rng, q.shape)))
        ws.fill_(255 - i)
        graph.replay()
        laq.paged_attention(q, k, v, table, start, lens, out=again, workspace=ws2)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), again.view(torch.int16)), i
        arrays = tuple(x.cpu().numpy() for x in (table, start, lens, k, v))
        check(out.cpu().numpy(), q.cpu().numpy(), arrays, 0, False)


def best_time(f, calls=3):
    """Shortest of some calls, in ms."""
    times = []
    for _ in range(calls + 1):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times[1:])


def decoding(B, Hq=2, Hkv=1):
    """B decoding sequences of 16 positions."""
    return (torch.zeros((B, Hkv, 16, 128), dtype=torch.float16, device=DEV),
            torch.zeros((B, Hkv, 16, 128), dtype=torch.float16, device=DEV),
            torch.arange(B, dtype=torch.int32, device=DEV)[:, None], torch.arange(B + 1, dtype=torch.int32, device=DEV),
            torch.full((B,), 16, dtype=torch.int32, device=DEV))


def test_append_time_grows_with_the_rows():
    """16 times the sequences take 16 times as long at most, as their bytes do,
    with as much again for the timing: each row's search of its sequence does
    not grow with their number (it took 256 times as long then)."""
    say("append time")
    times = []
    for B in (8192, 131072):
        k, v, table, start, lens = decoding(B)
        qkv = torch.zeros((B, 4 * 128), dtype=torch.float16, device=DEV)
        q = torch.zeros((B, 2, 128), dtype=torch.float16, device=DEV)
        cs = decode.rope_table(16, 1e6, DEV)
        times.append(best_time(lambda: laq.paged_append(qkv, None, None, cs, k, v, table, start, lens, 2, 1e-6, q_out=q)))
    assert times[1] < 32 * times[0], times


def test_attention_time_grows_with_the_sequences():
    """As for the append: the items' search of their sequences does not grow
    with the square of the batch."""
    say("attention time")
    times = []
    for B in (2048, 32768):
        k, v, table, start, lens = decoding(B)
        q = torch.zeros((B, 2, 128), dtype=torch.float16, device=DEV)
        out = torch.zeros_like(q)
        times.append(best_time(lambda: laq.paged_attention(q, k, v, table, start, lens, out=out)))
    assert times[1] < 32 * times[0], times


# ---------------------------------------------------------------------------
# layouts
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("tokens", [[1, 2], [40, 1]])
def test_strides_of_dimensions_of_one_element(tokens):
    """One page, one key/value head, one table column, of any strides: they do
    not matter, and neither do those of keys and values have to be equal there."""
    say("dimensions of one", tokens)
    rng = np.random.default_rng(3)
    Hq = 2
    start = dev(np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32))
    lens = dev(np.array(tokens, dtype=np.int32) + 3)
    T = sum(tokens)
    x = f16(rng, (2, 2, 64, 128))
    k = dev(x[0])[:, None]                                          # strides of one head: 8192
    v = dev(x[1])[:, :, None].transpose(1, 2)                       # and 128
    assert k.stride() != v.stride()
    column = dev(np.array([[1, 0]], dtype=np.int32)).t()            # [2][1], element stride 2
    assert column.stride() == (1, 2)
    q, qkv = f16(rng, (T, Hq, 128)), f16(rng, (T, (Hq + 2) * 128))
    cs = decode.rope_table(64, 1e6, DEV)
    plain = [dev(x[0][:, None]), dev(x[1][:, None]), dev(np.array([[1], [0]], dtype=np.int32)), start, lens]
    odd = [k, v, column, start, lens]
    outs = [laq.paged_append(dev(qkv), None, None, cs, *a, Hq, 1e-6) for a in (plain, odd)]
    outs += [laq.paged_attention(dev(q), *a) for a in (plain, odd)]
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[3])
    assert torch.equal(k, plain[0]) and torch.equal(v, plain[1])
    # one page whose stride is no multiple of 8
    one = torch.zeros((1, 1, 64, 128), dtype=torch.float16, device=DEV).as_strided((1, 1, 64, 128), (8195, 4, 128, 1))
    same = torch.zeros((1, 1, 64, 128), dtype=torch.float16, device=DEV)
    args = (dev(np.array([[0], [0]], dtype=np.int32)), start, lens)
    assert torch.equal(laq.paged_attention(dev(q), one, one, *args), laq.paged_attention(dev(q), same, same, *args))


@pytest.mark.parametrize("tokens", [[2, 1, 3], [2, 40, 30]])
def test_row_starts_outside_the_batch(tokens):
    """Row starts below 0 count as 0 and ones above T as T."""
    say("row starts outside", tokens)
    rng = np.random.default_rng(12)
    Hq, Hkv = 4, 2
    bt = Batch(rng, tokens, [30, 70, 9], 16, Hkv, garbage=None)
    q, qkv = f16(rng, (bt.T, Hq, 128)), f16(rng, (bt.T, (Hq + 2 * Hkv) * 128))
    cs = decode.rope_table(200, 1e6, DEV)
    got = []
    for start in (bt.start, np.array([-7, *bt.start[1:3], bt.T + 1000], dtype=np.int32),
                  np.array([-2**31, *bt.start[1:3], 2**31 - 1], dtype=np.int32)):
        k, v, table, _, lens = bt.device()
        rows = laq.paged_append(dev(qkv), None, None, cs, k, v, table, dev(start), lens, Hq, 1e-6)
        got.append((rows, k, v, laq.paged_attention(dev(q), k, v, table, dev(start), lens)))
    torch.cuda.synchronize()
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# few rows beside a chunk: the checks of decoding batches, in the kernel of chunks
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("tokens,before,window", [([1, 60], [100, 60], 0), ([4, 60], [90, 40], 48), ([8, 60], [700, 40], 0)])
def test_unseen_values_beside_a_chunk(tokens, before, window):
    unseen_values(tokens, before, window)


@pytest.mark.parametrize("tokens,before", [([2, 60], [700, 60]), ([3, 40], [30, 0])])
def test_not_finite_inputs_beside_a_chunk(tokens, before):
    not_finite_inputs(tokens, before)


def test_rows_that_see_nothing_beside_a_chunk():
    rows_that_see_nothing([4, 60, 3])
    rows_that_see_nothing([60, 2, 3])


def test_two_streams_at_once():
    """Calls in flight on two streams, workspaces taken from the allocator."""
    say("two streams")
    rng = np.random.default_rng(77)
    batches = [Batch(rng, *x, 16, 2) for x in (([1, 1, 2], [3000, 900, 40]), ([200, 1], [1500, 2500]))]
    qs = [f16(rng, (bt.T, 8, 128)) for bt in batches]
    alone = [attend(q, bt) for q, bt in zip(qs, batches)]
    args = [(dev(q), *bt.device()) for q, bt in zip(qs, batches)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(laq.paged_attention(*args[i]))
    torch.cuda.synchronize()
    for ref, outs in zip(alone, got):
        for out in outs:
            assert np.array_equal(out.cpu().numpy().view(np.uint16), ref.view(np.uint16))


# ---------------------------------------------------------------------------
# sampling: borders of its passes over a row
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("V", [7, 8, 9, 15, 16, 17, 8192, 8199, 40952, 40960, 40961, 49152, 81920, 81927, 122880])
def test_sample_borders_of_vectors(V):
    """Vectors of 8 logits, 8192 a pass of the block, 5 and 10 of them loaded
    ahead: the last token, the last of a vector and the first are drawn too."""
    say("sample borders", V)
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((6, V)) * 2).astype(np.float16)
    places = [V - 1, 0, V - 2, (V // 8 * 8 - 1) % V, min(8192, V) - 1]
    for r, t in enumerate(places):
        x[r, t] = np.float16(30)  # takes all
    u = rng.random(6).astype(np.float32)
    tok = sample_check(x, u)
    assert tok.tolist()[:5] == places
    sample_check(x, u, temperature=[5.0] * 6, top_k=[3, 0, V, V - 1, 10, 1], top_p=[0.9, 0.5, 1, 1, 0.99, 1])
    sample_check(x, u, temperature=[0.0] * 6)


@pytest.mark.parametrize("n", [1, 2, 1023, 1024, 1025, 2048, 4097])
def test_sample_equal_tokens(n):
    """The nth of so many tokens of one value, of which 1024 are listed."""
    say("sample equal tokens", n)
    V = 20011
    rng = np.random.default_rng(n)
    x = np.full((7, V), -np.inf, dtype=np.float16)
    for r in range(7):
        x[r, rng.permutation(V)[:n]] = np.float16(2.5)
    sample_check(x, np.array([0.0, 0.2, 0.5, 0.7, 0.999, 1.0, 1 / 3], dtype=np.float32))
    sample_check(x, np.full(7, 0.99, dtype=np.float32), top_k=[1, n, 1024, 1025, 0, n + 1, max(n - 1, 1)])
