"""Operators of batched serving as measurable cases, with their plain forms.

Three operators that take a batch of sequences from the q|k|v projection to
the next tokens:

  append     per-head RMSNorm of q and k, rotary embedding, and k and v
             written to a paged cache (laq.paged_append)
  attention  new tokens of several sequences over their paged caches, causal,
             optionally within a window (laq.paged_attention)
  sample     temperature, top-k, top-p and min-p sampling from given uniform
             numbers (laq.sample)

A batch: sequence b owns rows token_start[b] .. token_start[b + 1] - 1 of the
step's rows; its cache holds seq_len[b] positions, the new rows being the last
of them; position t lies in page page_table[b][t // page_size], slot t %
page_size.  Head dimension 128.

Head counts, vocabulary and sampling settings are those of the Qwen3 shapes in
`decode.py` and `inputs.py`, and generic ones.
"""
import math

import numpy as np
import torch

own = False  # whether run() calls the library's operators or their plain forms

DEV = "cuda:0"
HEAD = 128
EPS = 1e-6
THETA = 1e6
VOCAB = 151936


def _text(numbers):
    return " ".join(str(n) for n in numbers)


def _numbers(text):
    return [int(n) for n in text.split()]


def listed():
    return [
        # A decode step of 16 sequences (the linears' largest batch): one new
        # token each, latency.
        {"name": "append_decode16", "kind": "append", "heads": 32, "kv_heads": 8, "page": 16, "norm": True,
         "tokens": _text([1] * 16), "before": _text(range(7, 4016, 251)), "pad": 0, "slot_major": False},
        # Chunks of several prompts beside decoding sequences, odd lengths,
        # padding rows behind the last sequence, a model without q/k norms and
        # a cache whose pages hold position-major rows.
        {"name": "append_ragged", "kind": "append", "heads": 28, "kv_heads": 4, "page": 64, "norm": False,
         "tokens": "777 1 0 512 1 1 301 65 1", "before": "0 4097 33 1024 15 900 63 2000 1",
         "pad": 21, "slot_major": True},
        # Prompts of four requests at once.
        {"name": "append_prompts", "kind": "append", "heads": 32, "kv_heads": 8, "page": 128, "norm": True,
         "tokens": "8192 4001 2500 1691", "before": "0 0 512 0", "pad": 0, "slot_major": False},
        # One token of one sequence at a short context (32B heads): latency.
        {"name": "attention_one", "kind": "attention", "heads": 64, "kv_heads": 8, "page": 16, "window": 0,
         "tokens": "1", "before": "299", "pad": 0, "slot_major": False},
        # A decode step of 16 sequences of mixed lengths (4B heads).
        {"name": "attention_decode16", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 16, "window": 0,
         "tokens": _text([1] * 16),
         "before": "0 35 130 257 511 760 1023 1300 1999 2500 3011 4095 5000 6001 7100 8191", "pad": 0, "slot_major": False},
        # Two long documents being answered, and one short (32B heads).
        {"name": "attention_long", "kind": "attention", "heads": 64, "kv_heads": 8, "page": 64, "window": 0,
         "tokens": "1 1 1", "before": "131071 77776 900", "pad": 0, "slot_major": False},
        # A prompt taken in pieces of 16 rows (the linears' largest batch).
        {"name": "attention_chunk16", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 32, "window": 0,
         "tokens": "16", "before": "6000", "pad": 0, "slot_major": False},
        # A prompt's chunk beside decoding sequences, five query heads per
        # key/value head, a window whose expired pages were given back.
        {"name": "attention_mixed", "kind": "attention", "heads": 40, "kv_heads": 8, "page": 16, "window": 2048,
         "tokens": _text([500] + [1] * 15), "before": _text([3900] + [150 + 260 * i for i in range(15)]),
         "pad": 3, "slot_major": True},
        # Two fresh prompts (4B heads).
        {"name": "attention_prompts", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 64, "window": 0,
         "tokens": "8192 4001", "before": "0 0", "pad": 0, "slot_major": False},
        # The next token of one sequence: latency.
        {"name": "sample_one", "kind": "sample", "rows": 1, "vocab": VOCAB, "mix": "usual", "masked": 0.0},
        # 64 sequences, each with its own settings, greedy ones among them.
        {"name": "sample_batch64", "kind": "sample", "rows": 64, "vocab": VOCAB, "mix": "each", "masked": 0.0},
        # Many rows of an odd vocabulary, most of it masked (a grammar).
        {"name": "sample_odd256", "kind": "sample", "rows": 256, "vocab": 32003, "mix": "each", "masked": 0.7},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(1, 1), (8, 1), (14, 2), (16, 16), (28, 4), (32, 8), (32, 8), (40, 8), (64, 8), (48, 16)]


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "sample"])
    if kind == "sample":
        vocab = _log_int(rng, 500, VOCAB)
        rows = _log_int(rng, 1, min(256, 64 * VOCAB // vocab))
        return {"kind": kind, "rows": rows, "vocab": vocab, "mix": rng.choice(["usual", "each", "plain"]),
                "masked": rng.choice([0.0, 0.0, rng.uniform(0.1, 0.99)])}
    Hq, Hkv = rng.choice(_HEADS)
    case = {"kind": kind, "heads": Hq, "kv_heads": Hkv, "page": 2 ** rng.randint(4, 8),
            "slot_major": rng.random() < 0.3, "pad": rng.choice([0, 0, rng.randint(1, 40)])}
    if kind == "append":
        B = _log_int(rng, 1, 64)
        most = 16384 * 48 // (Hq + 2 * Hkv) // B
        top = _log_int(rng, 1, min(16384, most))
        tokens = [rng.randint(0, 1) if rng.random() < 0.3 else rng.randint(1, top) for _ in range(B)]
        before = [_log_int(rng, 1, 8192) - 1 for _ in range(B)]
        case["norm"] = rng.random() < 0.7
    else:
        B = _log_int(rng, 1, 32)
        if rng.random() < 0.5:  # decoding, a few rows per sequence at most
            tokens = [rng.choice([1, 1, 1, rng.randint(1, 4)]) for _ in range(B)]
            top = min(131072, 200000 * 8 // (B * Hkv))
            before = [_log_int(rng, 1, _log_int(rng, 16, top)) - 1 for _ in range(B)]
        else:  # chunks of prompts
            B = min(B, 8)
            # a padded batch's scores stay within those of the largest listed case
            n = _log_int(rng, 2, min(4096, int(math.sqrt(2**31 / (B * Hq)))))
            ctx = _log_int(rng, 1, min(16384, 2**31 // (B * Hq * n)))
            tokens = [n if i == 0 else rng.randint(1, n) for i in range(B)]
            before = [_log_int(rng, 1, ctx) - 1 for _ in range(B)]
        case["window"] = rng.choice([0, 0, _log_int(rng, 16, 4096)])
    if sum(tokens) == 0:
        tokens[0] = 1
    case["tokens"], case["before"] = _text(tokens), _text(before)
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1013 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _int32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _reach(case):
    """Positions of the longest sequence."""
    return max(n + p for n, p in zip(_numbers(case["tokens"]), _numbers(case["before"])))


def _batch(case, g):
    """page_table, token_start, seq_len and empty caches whose unused slots hold
    what freed memory holds (NaN among it, for attention, which must not read
    it)."""
    ps, Hkv = case["page"], case["kv_heads"]
    tokens, before = _numbers(case["tokens"]), _numbers(case["before"])
    lens = [n + p for n, p in zip(tokens, before)]
    pages = [(n + ps - 1) // ps for n in lens]
    width = max(max(pages), 1)
    spare = 3
    total = sum(pages) + spare
    order = torch.randperm(total, generator=g, device=DEV).cpu().numpy().astype(np.int32)
    table = np.full((len(tokens), width), -1, dtype=np.int32)
    used = np.zeros((total, ps), dtype=bool)
    at = 0
    for b, n in enumerate(pages):
        mine = order[at:at + n]
        at += n
        table[b, :n] = mine
        used[mine] = True
        if lens[b] % ps:
            used[mine[-1], lens[b] % ps:] = False
        w = case.get("window", 0)
        if w and n:  # pages that no new row sees any more were given back
            table[b, :max(0, before[b] - w + 1) // ps] = -1
    shape = (total, ps, Hkv, HEAD) if case["slot_major"] else (total, Hkv, ps, HEAD)
    st = {"case": case, "page_table": torch.from_numpy(table).to(DEV), "seq_len": _int32(lens),
          "token_start": _int32([0] + list(np.cumsum(tokens)))}
    for name in ("k_pages", "v_pages"):
        c = _randn(g, *shape).to(torch.float16)
        if case["kind"] == "attention":
            free = ~torch.from_numpy(used).to(DEV)
            c.masked_fill_(free[:, :, None, None] if case["slot_major"] else free[:, None, :, None], float("nan"))
        st[name] = c.transpose(1, 2) if case["slot_major"] else c
    return st


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] == "sample":
        st = {"case": case}
        st.update(_sample_inputs(case, g))
    else:
        st = _batch(case, g)
        Hq, Hkv = case["heads"], case["kv_heads"]
        rows = sum(_numbers(case["tokens"])) + case["pad"]
        if case["kind"] == "append":
            st["qkv"] = (1.5 * _randn(g, rows, (Hq + 2 * Hkv) * HEAD)).to(torch.float16)
            st["q_norm"], st["k_norm"] = (((1 + 0.1 * _randn(g, HEAD)).to(torch.float16) if case["norm"] else None)
                                          for _ in range(2))
            st["cos_sin"] = _rope_table(_reach(case))
            st["q"] = torch.zeros((rows, Hq, HEAD), dtype=torch.float16, device=DEV)
        else:
            st["q"] = (2 * _randn(g, rows, Hq, HEAD)).to(torch.float16)
            st["out"] = torch.zeros((rows, Hq, HEAD), dtype=torch.float16, device=DEV)
    torch.cuda.synchronize()
    return st


def _rope_table(n):
    """fp32 [n][128]: the cosines of the 64 angles of each position, their sines."""
    a = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * torch.pow(
        torch.tensor(THETA, dtype=torch.float64, device=DEV),
        -2.0 * torch.arange(64, dtype=torch.float64, device=DEV) / HEAD)
    return torch.cat([torch.cos(a), torch.sin(a)], dim=1).to(torch.float32)


def _sample_inputs(case, g):
    R, V = case["rows"], case["vocab"]
    # a model's logits: a broad bulk, a few candidates well above it
    x = 2.5 * _randn(g, R, V) - 2
    x += 12 * (torch.rand((R, V), generator=g, device=DEV) < 20.0 / V) * torch.rand((R, V), generator=g, device=DEV)
    if case["masked"]:
        x.masked_fill_(torch.rand((R, V), generator=g, device=DEV) < case["masked"], float("-inf"))
    uniform = lambda lo, hi: lo + (hi - lo) * torch.rand((R,), generator=g, device=DEV)  # noqa: E731
    pick = lambda p: torch.rand((R,), generator=g, device=DEV) < p  # noqa: E731
    st = {"logits": x.to(torch.float16), "u": uniform(0, 1)}
    if case["mix"] == "usual":
        st["temperature"], st["top_p"] = torch.full((R,), 0.6, device=DEV), torch.full((R,), 0.95, device=DEV)
        st["top_k"], st["min_p"] = torch.full((R,), 20, dtype=torch.int32, device=DEV), None
    elif case["mix"] == "plain":
        st["temperature"], st["top_k"], st["top_p"], st["min_p"] = torch.ones((R,), device=DEV), None, None, None
    else:
        zero = torch.zeros((R,), device=DEV)
        st["temperature"] = torch.where(pick(0.15), zero, uniform(0.3, 1.5))
        k = torch.exp(uniform(0, math.log(V))).to(torch.int32)
        st["top_k"] = torch.where(pick(0.5), k, torch.zeros_like(k))
        st["top_p"] = torch.where(pick(0.5), uniform(0.3, 0.999), zero + 1)
        st["min_p"] = torch.where(pick(0.3), uniform(0.0005, 0.2), zero)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if own:
        from paper_2605_08755_amd import laq
        if case["kind"] == "sample":
            return laq.sample(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"],
                              top_p=st["top_p"], min_p=st["min_p"])
        if case["kind"] == "append":
            laq.paged_append(st["qkv"], st["q_norm"], st["k_norm"], st["cos_sin"], st["k_pages"], st["v_pages"],
                             st["page_table"], st["token_start"], st["seq_len"], case["heads"], EPS, q_out=st["q"])
            return st["q"], st["k_pages"], st["v_pages"]
        return laq.paged_attention(st["q"], st["k_pages"], st["v_pages"], st["page_table"], st["token_start"],
                                   st["seq_len"], window=case["window"], out=st["out"])
    return {"sample": _sample, "append": _append, "attention": _attention}[case["kind"]](st)


def _row_places(st, rows):
    """Sequence and position of rows 0 .. rows - 1 (all of them some sequence's)."""
    start = st["token_start"].long()
    r = torch.arange(rows, device=DEV)
    b = torch.searchsorted(start[1:], r, right=True)
    return b, st["seq_len"].long()[b] - start[b + 1] + r


def _append(st):
    case = st["case"]
    Hq, Hkv, ps = case["heads"], case["kv_heads"], case["page"]
    rows = sum(_numbers(case["tokens"]))
    x = st["qkv"][:rows].view(rows, Hq + 2 * Hkv, HEAD)
    b, pos = _row_places(st, rows)
    qk = x[:, :Hq + Hkv].float()
    if case["norm"]:
        w = torch.cat([st["q_norm"].expand(Hq, HEAD), st["k_norm"].expand(Hkv, HEAD)]).float()
        qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * w
    c, s = st["cos_sin"][pos][:, None].split(64, dim=-1)
    a, e = qk.split(64, dim=-1)
    qk = torch.cat([a * c - e * s, e * c + a * s], dim=-1).to(torch.float16)
    page, slot = st["page_table"][b, pos // ps].long(), pos % ps
    st["q"][:rows] = qk[:, :Hq]
    st["k_pages"][page, :, slot] = qk[:, Hq:]
    st["v_pages"][page, :, slot] = x[:, Hq + Hkv:]
    return st["q"], st["k_pages"], st["v_pages"]


def _attention(st):
    """The batch padded to its longest sequence and its largest chunk."""
    case = st["case"]
    Hq, Hkv, ps = case["heads"], case["kv_heads"], case["page"]
    tokens = _numbers(case["tokens"])
    B, N, L, rows, R = len(tokens), max(tokens), _reach(case), sum(tokens), Hq // Hkv
    start, lens = st["token_start"].long(), st["seq_len"].long()
    t = torch.arange(L, device=DEV)
    page = st["page_table"].long()[:, t // ps]
    there = (page >= 0) & (t < lens[:, None])
    at = page.clamp(min=0)

    def rows_of(cache):  # [B][Hkv][L][128], zeros where nothing is
        x = cache[at, :, t % ps]
        return torch.where(there[:, :, None, None], x, torch.zeros((), dtype=x.dtype, device=DEV)).transpose(1, 2)
    n = torch.arange(N, device=DEV)
    r = (start[:-1, None] + n).clamp(max=rows - 1)
    q = st["q"][r].float().view(B, N, Hkv, R, HEAD).permute(0, 2, 3, 1, 4).reshape(B, Hkv, R * N, HEAD)
    s = torch.matmul(q, rows_of(st["k_pages"]).float().transpose(2, 3).contiguous()) * (1 / math.sqrt(HEAD))
    pos = (lens - (start[1:] - start[:-1]))[:, None] + n
    sees = there[:, None] & (t <= pos[:, :, None])
    if case["window"]:
        sees &= t > pos[:, :, None] - case["window"]
    s = s.view(B, Hkv, R, N, L).masked_fill_(~sees[:, None, None], float("-inf"))
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = s.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, R * N, L), rows_of(st["v_pages"]).float().contiguous()).view(B, Hkv, R, N, HEAD)
    o = torch.where(z > 0, o / z, torch.zeros((), device=DEV))
    b, _ = _row_places(st, rows)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, N, Hq, HEAD)
    st["out"][:rows] = o[b, torch.arange(rows, device=DEV) - start[b]].to(torch.float16)
    return st["out"]


def _sample(st):
    x = st["logits"]
    R, V = x.shape
    x = torch.where(torch.isnan(x), torch.full((), float("-inf"), dtype=x.dtype, device=DEV), x)
    v, order = torch.sort(x, dim=1, descending=True, stable=True)
    m = v[:, :1].double()
    temp = st["temperature"].double()[:, None] if st["temperature"] is not None else torch.ones_like(m)
    greedy = ~(temp > 0)
    d = torch.where(v == v[:, :1], torch.zeros((), dtype=torch.float64, device=DEV), v.double() - m)
    w = torch.exp(d / torch.where(greedy, torch.ones_like(temp), temp))  # 64 bits: neighbours of a long running sum
    i = torch.arange(V, device=DEV)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        w = torch.where((i < k) | (k <= 0), w, 0.0)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        c = torch.cumsum(w, dim=1)
        before = torch.cat([torch.zeros_like(m), c[:, :-1]], dim=1)
        kept = (before < p * c[:, -1:]) | ~(p < 1) | (i == 0)
    else:
        kept = torch.ones_like(w, dtype=torch.bool)
    if st["min_p"] is not None:
        kept &= (w >= st["min_p"].double()[:, None].clamp(max=1))
    w = torch.where(kept, w, 0.0)
    c = torch.cumsum(w, dim=1)
    past = c > st["u"].double()[:, None] * c[:, -1:]
    at = torch.where(past.any(1), past.int().argmax(1), (w > 0).sum(1) - 1)[:, None]
    at = torch.where(greedy, torch.zeros_like(at), at)
    prob = torch.where(greedy, torch.ones_like(m), torch.gather(w, 1, at) / c[:, -1:])
    none = torch.isneginf(m)
    token = torch.where(none, torch.full_like(at, -1), torch.gather(order, 1, at))
    return token[:, 0].to(torch.int32), torch.where(none, torch.zeros_like(prob), prob)[:, 0].to(torch.float32)


# ---------------------------------------------------------------------------
# work
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": 2.0 * n + 28 * case["rows"], "flops": 4.0 * n}
    tokens, before = _numbers(case["tokens"]), _numbers(case["before"])
    Hq, Hkv, ps, rows = case["heads"], case["kv_heads"], case["page"], sum(tokens)
    if case["kind"] == "append":
        # every head of every row in and out, the table's rows that positions share
        return {"bytes": 2.0 * rows * (Hq + 2 * Hkv) * HEAD * 2 + 512.0 * min(rows, _reach(case)) + 8 * rows,
                "flops": 10.0 * rows * (Hq + Hkv) * HEAD}
    w = case["window"]
    seen, pairs = 0, 0
    for n, p in zip(tokens, before):
        if n == 0:
            continue
        first = max(0, p - w + 1) if w else 0
        seen += n + p - first
        if w:
            pairs += sum(min(w, p + j + 1) for j in range(n))
        else:
            pairs += n * p + n * (n + 1) // 2
    return {"bytes": 4.0 * seen * Hkv * HEAD + 4.0 * rows * Hq * HEAD + 4.0 * seen / ps + 8.0 * len(tokens),
            "flops": 4.0 * HEAD * Hq * pairs}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(st)
    starts = np.concatenate([[0], np.cumsum(_numbers(case["tokens"]))]).tolist()
    table = st["page_table"].tolist()
    return (_exact_append if case["kind"] == "append" else _exact_attention)(case, st, starts, table)


def _places(case, table, b, lo, hi):
    """Pages and slots of positions lo .. hi - 1 of sequence b."""
    t = range(lo, hi)
    ps = case["page"]
    return (torch.tensor([table[b][i // ps] for i in t], device=DEV, dtype=torch.long),
            torch.tensor([i % ps for i in t], device=DEV, dtype=torch.long))


def _exact_append(case, st, starts, table):
    Hq, Hkv = case["heads"], case["kv_heads"]
    q, kc, vc = st["q"].double(), st["k_pages"].double(), st["v_pages"].double()
    freq = THETA ** (-np.arange(64) / 64.0)
    for b, (n, p) in enumerate(zip(_numbers(case["tokens"]), _numbers(case["before"]))):
        if n == 0:
            continue
        angle = torch.from_numpy(np.outer(np.arange(p, p + n), freq)).to(DEV)
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]  # pairs as complex numbers
        x = st["qkv"][starts[b]:starts[b + 1]].double().view(n, -1, HEAD)
        done = []
        for part, w in ((x[:, :Hq], st["q_norm"]), (x[:, Hq:Hq + Hkv], st["k_norm"])):
            if w is not None:
                part = part / (part.square().sum(-1, keepdim=True) / HEAD + EPS).sqrt() * w.double()
            z = torch.complex(part[..., :64].contiguous(), part[..., 64:].contiguous()) * turn
            done.append(torch.cat([z.real, z.imag], dim=-1))
        page, slot = _places(case, table, b, p, p + n)
        q[starts[b]:starts[b + 1]] = done[0]
        kc[page, :, slot] = done[1]
        vc[page, :, slot] = x[:, Hq + Hkv:]
    return q, kc, vc


def _exact_attention(case, st, starts, table):
    Hq, Hkv, w = case["heads"], case["kv_heads"], case["window"]
    R = Hq // Hkv
    out = st["out"].double()
    for b, (n, p) in enumerate(zip(_numbers(case["tokens"]), _numbers(case["before"]))):
        if n == 0:
            continue
        first = max(0, p - w + 1) if w else 0
        page, slot = _places(case, table, b, first, p + n)
        for g in range(Hkv):
            K, V = (st[c][page, g, slot].double() for c in ("k_pages", "v_pages"))
            step = max(1, 2**27 // (R * (p + n - first)))
            for j in range(0, n, step):
                e = min(n, j + step)
                # row j sees positions up to p + j: none of the rows here sees past p + e
                hi = p + e - first
                lo = max(0, p + j - w + 1 - first) if w else 0
                at = torch.arange(first + lo, first + hi, device=DEV)
                mine = torch.arange(p + j, p + e, device=DEV)[:, None]
                hide = (at > mine) | ((at <= mine - w) if w else torch.zeros_like(at, dtype=torch.bool))
                q = st["q"][starts[b] + j:starts[b] + e, g * R:(g + 1) * R].double().transpose(0, 1)
                s = (q.reshape(-1, HEAD) @ K[lo:hi].t().contiguous() / HEAD**0.5).view(R, e - j, -1)
                a = torch.softmax(s.masked_fill_(hide, -math.inf), dim=-1)
                out[starts[b] + j:starts[b] + e, g * R:(g + 1) * R] = (
                    a.view(R * (e - j), -1) @ V[lo:hi]).view(R, e - j, HEAD).transpose(0, 1)
    return out


def _exact_sample(st):
    """Row by row in numpy.  The drawn token is a whole number; its probability
    is the computed one."""
    x = st["logits"].cpu().numpy().astype(np.float64)
    R, V = x.shape
    setting = {n: st[n].double().cpu().numpy() if st[n] is not None else None
               for n in ("u", "temperature", "top_k", "top_p", "min_p")}
    tokens, probs = [], []
    for r in range(R):
        get = lambda n, off: off if setting[n] is None else float(setting[n][r])  # noqa: E731
        l = np.where(np.isnan(x[r]), -np.inf, x[r])
        top = l.max()
        if top == -np.inf:
            tokens.append(-1)
            probs.append(0.0)
            continue
        T = get("temperature", 1.0)
        if not T > 0:
            tokens.append(int(l.argmax()))
            probs.append(1.0)
            continue
        order = np.lexsort((np.arange(V), -l))
        w = np.exp((l[order] - top) / T)
        k = int(get("top_k", 0))
        if 0 < k < V:
            w = w[:k]
        n = len(w)
        p = get("top_p", 1.0)
        if p < 1:
            n = min(n, int(np.searchsorted(np.cumsum(w), p * math.fsum(w), side="left")) + 1)
        mp = get("min_p", 0.0)
        if mp > 0:
            n = min(n, int((w >= min(mp, 1.0)).sum()))
        w = w[:max(n, 1)]
        i = min(int(np.searchsorted(np.cumsum(w), get("u", 0.0) * math.fsum(w), side="right")), len(w) - 1)
        tokens.append(int(order[i]))
        probs.append(float(w[i] / math.fsum(w)))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64)
