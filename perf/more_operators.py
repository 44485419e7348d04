"""Operators of batched serving with caches in 8 bits, and of logits before
sampling, as measurable cases, with their plain forms.

  append     per-head RMSNorm of q and k, rotary embedding, and k and v written
             to paged caches in e4m3 with a scale for each 16 positions of a
             head (laq.paged_append_e4m3)
  attention  new tokens of several sequences over such caches, causal,
             optionally within a window (laq.paged_attention_e4m3)
  adjust     repetition, frequency and presence penalties, biases of listed
             tokens and a grammar's mask on the logits (laq.adjust_logits)

A batch: sequence b owns rows token_start[b] .. token_start[b + 1] - 1 of the
step's rows; its cache holds seq_len[b] positions, the new rows being the last
of them; position t lies in page page_table[b][t // page_size], slot t %
page_size.  Head dimension 128.

A cache holds the value code * 2^e, code in e4m3 and e that of the position's
block of 16, one for keys and one for values of a head.  Appending to a block
takes the least e in -15..7 for which 448 * 2^e holds its new values, but none
below the one that its earlier positions have; these are rounded again where it
grows.
"""
import math

import numpy as np
import torch

own = False  # whether run() calls the library's operators or their plain forms

DEV = "cuda:0"
HEAD = 128
BLOCK = 16
EPS = 1e-6
THETA = 1e6
VOCAB = 151936
LOWEST, HIGHEST = 112, 134  # exponents -15 and 7, as an e8m0 scale has them


def _text(numbers):
    return " ".join(str(n) for n in numbers)


def _numbers(text):
    return [int(n) for n in text.split()]


def listed():
    return [
        # A decode step of 16 sequences (the linears' largest batch), most of
        # whose blocks hold earlier positions: latency.
        {"name": "append8_decode16", "kind": "append", "heads": 32, "kv_heads": 8, "page": 16, "norm": True,
         "tokens": _text([1] * 16), "before": _text(range(7, 4016, 251)), "pad": 0, "slot_major": False},
        # Chunks of several prompts beside decoding and waiting sequences, odd
        # lengths, padding rows, no q/k norms, position-major pages.
        {"name": "append8_ragged", "kind": "append", "heads": 28, "kv_heads": 4, "page": 64, "norm": False,
         "tokens": "777 1 0 512 1 1 301 65 1", "before": "0 4097 33 1024 15 900 63 2000 1",
         "pad": 21, "slot_major": True},
        # Prompts of four requests at once.
        {"name": "append8_prompts", "kind": "append", "heads": 32, "kv_heads": 8, "page": 128, "norm": True,
         "tokens": "8192 4001 2500 1691", "before": "0 0 512 0", "pad": 0, "slot_major": False},
        # One token of one sequence at a short context (32B heads): latency.
        {"name": "attention8_one", "kind": "attention", "heads": 64, "kv_heads": 8, "page": 16, "window": 0,
         "tokens": "1", "before": "299", "pad": 0, "slot_major": False},
        # A decode step of 16 sequences of mixed lengths (4B heads).
        {"name": "attention8_decode16", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 16, "window": 0,
         "tokens": _text([1] * 16),
         "before": "0 35 130 257 511 760 1023 1300 1999 2500 3011 4095 5000 6001 7100 8191", "pad": 0, "slot_major": False},
        # Long documents being answered, and a short one (32B heads): what a
        # cache of half the bytes is for.
        {"name": "attention8_long", "kind": "attention", "heads": 64, "kv_heads": 8, "page": 64, "window": 0,
         "tokens": "1 1 1 1", "before": "131071 77776 120001 900", "pad": 0, "slot_major": False},
        # A prompt's chunk beside decoding sequences, five query heads per
        # key/value head, a window whose expired pages were given back.
        {"name": "attention8_mixed", "kind": "attention", "heads": 40, "kv_heads": 8, "page": 16, "window": 2048,
         "tokens": _text([500] + [1] * 15), "before": _text([3900] + [150 + 260 * i for i in range(15)]),
         "pad": 3, "slot_major": True},
        # Two fresh prompts (4B heads).
        {"name": "attention8_prompts", "kind": "attention", "heads": 32, "kv_heads": 8, "page": 64, "window": 0,
         "tokens": "8192 4001", "before": "0 0", "pad": 0, "slot_major": False},
        # The next token of one sequence in the middle of an answer: latency.
        {"name": "adjust_one", "kind": "adjust", "rows": 1, "vocab": VOCAB, "history": 700, "bias": 0, "mask": "none"},
        # 64 sequences, each with its own penalties, history and biases.
        {"name": "adjust_batch64", "kind": "adjust", "rows": 64, "vocab": VOCAB, "history": 8192, "bias": 20, "mask": "none"},
        # Grammars over an odd vocabulary, many rows.
        {"name": "adjust_grammar256", "kind": "adjust", "rows": 256, "vocab": 32003, "history": 2000, "bias": 300, "mask": "each"},
        # Long documents whose tokens all count as seen.
        {"name": "adjust_long16", "kind": "adjust", "rows": 16, "vocab": VOCAB, "history": 131072, "bias": 0, "mask": "one"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(1, 1), (8, 1), (14, 2), (16, 16), (28, 4), (32, 8), (32, 8), (40, 8), (64, 8), (48, 16)]


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "adjust"])
    if kind == "adjust":
        vocab = _log_int(rng, 500, VOCAB)
        rows = _log_int(rng, 1, min(256, 64 * VOCAB // vocab))
        return {"kind": kind, "rows": rows, "vocab": vocab, "history": _log_int(rng, 1, min(131072, 2**21 // rows)),
                "bias": rng.choice([0, 0, _log_int(rng, 1, 1000)]), "mask": rng.choice(["none", "one", "each"])}
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
    g.manual_seed(int(seed) * 1013 + 31)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV, dtype=torch.float32)


def _int32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _reach(case):
    """Positions of the longest sequence."""
    return max(n + p for n, p in zip(_numbers(case["tokens"]), _numbers(case["before"])))


def _two_to(e):
    """2^(e - 127) of whole numbers e in 1 .. 254, fp32."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _least(a):
    """The least exponent (as a scale has it) for which 448 times its power of two is a (fp32) or more."""
    return (((a.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(LOWEST, HIGHEST)


def _codes(x):
    """e4m3 of fp32 values: saturated, NaN where not finite."""
    x = torch.where(torch.isfinite(x), x.clamp(-448, 448), torch.full((), float("nan"), device=DEV))
    return x.to(torch.float8_e4m3fn)


def _batch(case, g):
    """page_table, token_start, seq_len and filled caches; what freed memory
    holds in their unused slots (NaN among it, for attention, which must not
    read it)."""
    ps, Hkv = case["page"], case["kv_heads"]
    tokens, before = _numbers(case["tokens"]), _numbers(case["before"])
    lens = [n + p for n, p in zip(tokens, before)]
    pages = [max((n + ps - 1) // ps, 1) for n in lens]
    total = sum(pages) + 3
    order = torch.randperm(total, generator=g, device=DEV).cpu().numpy().astype(np.int32)
    table = np.full((len(tokens), max(pages)), -1, dtype=np.int32)
    used = np.zeros((total, ps), dtype=bool)
    at = 0
    for b, n in enumerate(pages):
        mine = order[at:at + n]
        at += n
        table[b, :n] = mine
        used[mine] = True
        used[mine[-1], lens[b] - (n - 1) * ps:] = False
        w = case.get("window", 0)
        if w:  # pages that no new row sees any more were given back
            table[b, :max(0, before[b] - w + 1) // ps] = -1
    st = {"case": case, "page_table": torch.from_numpy(table).to(DEV), "seq_len": _int32(lens),
          "token_start": _int32([0] + list(np.cumsum(tokens)))}
    free = ~torch.from_numpy(used).to(DEV)[:, None, :, None]
    for name in ("k", "v"):
        x = _randn(g, total, Hkv, ps, HEAD)
        # some rows are larger than others, and of keys some dimensions
        x *= torch.exp(0.7 * _randn(g, total, Hkv, ps, 1))
        if name == "k":
            x *= torch.exp(0.8 * _randn(g, 1, Hkv, 1, HEAD))
        blocks = x.view(total, Hkv, ps // BLOCK, BLOCK * HEAD)
        e = _least(blocks.abs().amax(-1))
        codes = _codes((blocks / _two_to(e)[..., None]).view(total, Hkv, ps, HEAD)).view(torch.uint8)
        if case["kind"] == "attention":
            codes.masked_fill_(free, 0x7F)
        st[name + "_scales"] = e.to(torch.uint8).view(torch.float8_e8m0fnu)
        if case["slot_major"]:
            codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
        st[name + "_pages"] = codes.view(torch.float8_e4m3fn)
    return st


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] == "adjust":
        st = {"case": case}
        st.update(_adjust_inputs(case, g))
    else:
        st = _batch(case, g)
        Hq, Hkv = case["heads"], case["kv_heads"]
        rows = sum(_numbers(case["tokens"])) + case["pad"]
        if case["kind"] == "append":
            x = _randn(g, rows, Hq + 2 * Hkv, HEAD) * torch.exp(0.7 * _randn(g, rows, Hq + 2 * Hkv, 1))
            st["qkv"] = x.view(rows, -1).to(torch.float16)
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


def _adjust_inputs(case, g):
    R, V, H, N = case["rows"], case["vocab"], case["history"], case["bias"]
    # a model's logits: a broad bulk, a few candidates well above it
    x = 2.5 * _randn(g, R, V) - 2
    x += 12 * (_rand(g, R, V) < 20.0 / V) * _rand(g, R, V)
    # text: few tokens make most of it
    st = {"logits": x.to(torch.float16), "history": (V * _rand(g, R, H) ** 2).to(torch.int32).clamp(max=V - 1)}
    n = (H * _rand(g, R)).to(torch.int32) + 1
    n[0] = H
    st["history_len"], st["prompt_len"] = n, (n * _rand(g, R)).to(torch.int32)
    off = lambda p, x, none: torch.where(_rand(g, R) < p, torch.full_like(x, none), x)  # noqa: E731
    st["repetition"] = off(0.3, 0.9 + 0.5 * _rand(g, R), 1.0)
    st["frequency"] = off(0.5, 2 * _rand(g, R) - 0.5, 0.0)
    st["presence"] = off(0.5, 2 * _rand(g, R) - 0.5, 0.0)
    st["bias_token"] = st["bias_value"] = st["mask"] = None
    if N:
        t = (V * _rand(g, R, N)).to(torch.int32).clamp(max=V - 1)
        st["bias_token"] = torch.where(_rand(g, R, N) < 0.2, torch.full_like(t, -1), t)  # rows list fewer
        st["bias_value"] = torch.where(_rand(g, R, N) < 0.1, torch.full((), float("-inf"), device=DEV), 5 * _randn(g, R, N))
    if case["mask"] != "none":
        words = (V + 31) // 32
        rows = R if case["mask"] == "each" else 1  # one grammar for all rows
        m = (4294967296 * torch.rand((rows, words), generator=g, device=DEV, dtype=torch.float64)).to(torch.int64)
        m &= (4294967296 * torch.rand((rows, words), generator=g, device=DEV, dtype=torch.float64)).to(torch.int64)
        m = torch.where(_rand(g, rows, words) < 0.5, torch.zeros_like(m), m)
        st["mask"] = torch.where(m >= 2**31, m - 2**32, m).to(torch.int32).expand(R, words)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
_ADJUST = ("history", "history_len", "prompt_len", "repetition", "frequency", "presence", "bias_token", "bias_value", "mask")


def run(st):
    case = st["case"]
    if own:
        from paper_2605_08755_amd import laq
        if case["kind"] == "adjust":
            return laq.adjust_logits(st["logits"], **{n: st[n] for n in _ADJUST})
        if case["kind"] == "append":
            laq.paged_append_e4m3(st["qkv"], st["q_norm"], st["k_norm"], st["cos_sin"], st["k_pages"], st["v_pages"],
                                  st["k_scales"], st["v_scales"], st["page_table"], st["token_start"], st["seq_len"],
                                  case["heads"], EPS, q_out=st["q"])
            return st["q"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"]
        return laq.paged_attention_e4m3(st["q"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"],
                                        st["page_table"], st["token_start"], st["seq_len"], window=case["window"],
                                        out=st["out"])
    return {"adjust": _adjust, "append": _append, "attention": _attention}[case["kind"]](st)


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
    qk = torch.cat([a * c - e * s, e * c + a * s], dim=-1)
    st["q"][:rows] = qk[:, :Hq].to(torch.float16)
    page, slot = st["page_table"][b, pos // ps].long(), pos % ps
    # the block in which each sequence's new positions begin (of a waiting one, some block of its own)
    n = st["token_start"][1:].long() - st["token_start"][:-1].long()
    at = (st["seq_len"].long() - n).clamp(max=st["page_table"].shape[1] * ps - 1)
    at = torch.where(n > 0, at, (at - 1).clamp(min=0))
    kept = torch.where(n > 0, at % BLOCK, torch.full_like(at, BLOCK))  # its earlier positions
    first = st["page_table"][torch.arange(len(n), device=DEV), at // ps].long()
    _store(st["k_pages"], st["k_scales"], qk[:, Hq:], page, slot, first, at % ps // BLOCK, kept)
    _store(st["v_pages"], st["v_scales"], x[:, Hq + Hkv:].float(), page, slot, first, at % ps // BLOCK, kept)
    return st["q"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"]


def _store(pages, scales, x, page, slot, first, first_block, kept):
    P, Hkv, ps, _ = pages.shape
    codes, e_old = pages.view(torch.uint8), scales.view(torch.uint8)
    blocks = ps // BLOCK
    mine, lead = page * blocks + slot // BLOCK, first * blocks + first_block
    e_was = e_old.transpose(1, 2).reshape(P * blocks, Hkv).int()
    size = torch.where(torch.isfinite(x), x.abs(), torch.zeros((), device=DEV)).amax(-1)
    size = torch.zeros((P * blocks, Hkv), device=DEV).scatter_reduce_(0, mine[:, None].expand(-1, Hkv), size, "amax")
    e = _least(size)
    floor = torch.full_like(e, LOWEST)
    floor[lead] = torch.where((kept > 0)[:, None], e_was[lead], LOWEST)
    touched = torch.zeros((P * blocks, 1), dtype=torch.bool, device=DEV)
    touched[mine] = True
    e = torch.where(touched, torch.maximum(e, floor), e_was)
    e_old.copy_(e.view(P, blocks, Hkv).transpose(1, 2))
    # earlier positions of the first blocks
    slots = first_block[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    was = codes[first[:, None], :, slots]  # [B][16][Hkv][128]
    again = was.view(torch.float8_e4m3fn).float() * (_two_to(e_was[lead]) / _two_to(e[lead]))[:, None, :, None]
    keep = torch.arange(BLOCK, device=DEV)[None, :, None, None] >= kept[:, None, None, None]
    codes[first[:, None], :, slots] = torch.where(keep, was, again.to(torch.float8_e4m3fn).view(torch.uint8))
    codes[page, :, slot] = _codes(x / _two_to(e[mine])[..., None]).view(torch.uint8)


def _values(pages, scales, at, slot):
    """fp32 values of positions: pages' numbers and slots -> [..][Hkv][128]."""
    x = pages.view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float()
    return x * _two_to(scales.view(torch.uint8)[at, :, slot // BLOCK])[..., None]


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

    def rows_of(name):  # [B][Hkv][L][128], zeros where nothing is
        x = _values(st[name + "_pages"], st[name + "_scales"], at, (t % ps).expand(B, L))
        return torch.where(there[:, :, None, None], x, torch.zeros((), device=DEV)).transpose(1, 2)
    n = torch.arange(N, device=DEV)
    r = (start[:-1, None] + n).clamp(max=rows - 1)
    q = st["q"][r].float().view(B, N, Hkv, R, HEAD).permute(0, 2, 3, 1, 4).reshape(B, Hkv, R * N, HEAD)
    s = torch.matmul(q, rows_of("k").transpose(2, 3).contiguous()) * (1 / math.sqrt(HEAD))
    pos = (lens - (start[1:] - start[:-1]))[:, None] + n
    sees = there[:, None] & (t <= pos[:, :, None])
    if case["window"]:
        sees &= t > pos[:, :, None] - case["window"]
    s = s.view(B, Hkv, R, N, L).masked_fill_(~sees[:, None, None], float("-inf"))
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = s.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, R * N, L), rows_of("v").contiguous()).view(B, Hkv, R, N, HEAD)
    o = torch.where(z > 0, o / z, torch.zeros((), device=DEV))
    b, _ = _row_places(st, rows)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, N, Hq, HEAD)
    st["out"][:rows] = o[b, torch.arange(rows, device=DEV) - start[b]].to(torch.float16)
    return st["out"]


def _adjust(st):
    x = st["logits"].float()
    R, V = x.shape
    i = torch.arange(st["history"].shape[1], device=DEV)
    there = i < st["history_len"][:, None]
    told = st["history"].long()
    zero = torch.zeros((R, V), device=DEV)
    seen = zero.scatter_add(1, told, there.float())
    count = zero.scatter_add(1, told, (there & (i >= st["prompt_len"][:, None])).float())
    rep = st["repetition"][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - st["frequency"][:, None] * count - st["presence"][:, None] * (count > 0)
    if st["bias_token"] is not None:
        t = st["bias_token"].long()
        n = torch.arange(1, t.shape[1] + 1, device=DEV).expand_as(t)
        last = torch.zeros((R, V + 1), dtype=torch.int64, device=DEV).scatter_reduce_(
            1, torch.where(t >= 0, t, V), n, "amax")[:, :V]  # the last that lists a token counts
        x = torch.where(last > 0, x + torch.gather(st["bias_value"], 1, (last - 1).clamp(min=0)), x)
    if st["mask"] is not None:
        v = torch.arange(V, device=DEV)
        x = torch.where((st["mask"][:, v // 32] >> (v % 32)) & 1 == 1, x, float("-inf"))
    return x.to(torch.float16)


# ---------------------------------------------------------------------------
# work
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "adjust":
        R, V = case["rows"], case["vocab"]
        words = {"none": 0, "one": 1, "each": R}[case["mask"]] * ((V + 31) // 32)
        told = (R + 1) / 2 * case["history"]  # about half of each row's room, the first row's all
        return {"bytes": 4.0 * R * V + 4.0 * words + 4.0 * told + 8.0 * R * case["bias"], "flops": 4.0 * R * V}
    tokens, before = _numbers(case["tokens"]), _numbers(case["before"])
    Hq, Hkv, ps, rows = case["heads"], case["kv_heads"], case["page"], sum(tokens)
    if case["kind"] == "append":
        # every head of every row in, q out in 16 bits, k and v in 8 with their scales, the table's rows that positions share
        return {"bytes": 2.0 * rows * (2 * Hq + 2 * Hkv) * HEAD + rows * 2 * Hkv * (HEAD + 1 / BLOCK) +
                512.0 * min(rows, _reach(case)) + 8 * rows,
                "flops": 10.0 * rows * (Hq + Hkv) * HEAD + 6.0 * rows * Hkv * HEAD}
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
    return {"bytes": 2.0 * seen * Hkv * (HEAD + 1 / BLOCK) + 4.0 * rows * Hq * HEAD + 4.0 * seen / ps + 8.0 * len(tokens),
            "flops": 4.0 * HEAD * Hq * pairs}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "adjust":
        return _exact_adjust(st)
    starts = np.concatenate([[0], np.cumsum(_numbers(case["tokens"]))]).tolist()
    table = st["page_table"].tolist()
    return (_exact_append if case["kind"] == "append" else _exact_attention)(case, st, starts, table)


def _places(case, table, b, lo, hi):
    """Pages and slots of positions lo .. hi - 1 of sequence b."""
    t = range(lo, hi)
    ps = case["page"]
    return (torch.tensor([table[b][i // ps] for i in t], device=DEV, dtype=torch.long),
            torch.tensor([i % ps for i in t], device=DEV, dtype=torch.long))


def _held(pages, scales):
    """(codes, exponents) of a cache in 64 bits."""
    return pages.double(), scales.view(torch.uint8).long() - 127


def _exact_append(case, st, starts, table):
    """Codes before their rounding to e4m3 (those of positions that the call
    does not write as they are)."""
    Hq, Hkv, ps = case["heads"], case["kv_heads"], case["page"]
    q = st["q"].double()
    caches = [_held(st["k_pages"], st["k_scales"]), _held(st["v_pages"], st["v_scales"])]
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
        q[starts[b]:starts[b + 1]] = done[0]
        # positions of whole blocks: room for the earlier ones of the first and for those after the last
        lead, blocks = p % BLOCK, (p + n + BLOCK - 1) // BLOCK - p // BLOCK
        page, slot = _places(case, table, b, p, p + n)
        at_page, at_slot = _places(case, table, b, p - lead, p + n)
        heads = at_page[::BLOCK], at_slot[::BLOCK] // BLOCK
        for (codes, e), new in zip(caches, (done[1], x[:, Hq + Hkv:])):
            room = torch.zeros((blocks * BLOCK, Hkv, HEAD), dtype=torch.float64, device=DEV)
            room[lead:lead + n] = new
            size = room.view(blocks, BLOCK, Hkv, HEAD).abs().amax((1, 3)).cpu().numpy()
            least = np.ceil(np.log2(np.maximum(size, 1e-300) / 448))
            least += np.ldexp(448.0, least.astype(int)) < size  # where the logarithm is rounded
            least -= np.ldexp(448.0, least.astype(int) - 1) >= size
            least = torch.from_numpy(np.clip(least, -15, 7)).to(DEV).long()
            if lead:
                was = e[heads[0][0], :, heads[1][0]]
                least[0] = torch.maximum(least[0], was)
                codes[at_page[:lead], :, at_slot[:lead]] *= torch.pow(2.0, (was - least[0]).double())[None, :, None]
            e[heads[0], :, heads[1]] = least
            mine = least.repeat_interleave(BLOCK, dim=0)[lead:lead + n]
            codes[page, :, slot] = (new / torch.pow(2.0, mine.double())[..., None]).clamp(-448, 448)
    (kc, ke), (vc, ve) = caches
    return q, kc, vc, torch.pow(2.0, ke.double()), torch.pow(2.0, ve.double())


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
            K, V = (torch.ldexp(st[c + "_pages"].view(torch.uint8)[page, g, slot].view(torch.float8_e4m3fn).double(),
                                (st[c + "_scales"].view(torch.uint8)[page, g, slot // BLOCK].int() - 127)[:, None])
                    for c in ("k", "v"))
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


def _exact_adjust(st):
    """Row by row in numpy."""
    host = {n: None if st[n] is None else st[n].cpu().numpy() for n in ("logits",) + _ADJUST}
    V = host["logits"].shape[1]
    out = []
    for r, x in enumerate(host["logits"].astype(np.float64)):
        told = host["history"][r, :host["history_len"][r]]
        seen = np.unique(told)
        rep = float(host["repetition"][r])
        x[seen] = np.where(x[seen] > 0, x[seen] / rep, x[seen] * rep)
        count = np.bincount(told[host["prompt_len"][r]:], minlength=V)
        x -= float(host["frequency"][r]) * count + float(host["presence"][r]) * (count > 0)
        if host["bias_token"] is not None:
            told = dict(zip(host["bias_token"][r].tolist(), host["bias_value"][r].tolist()))
            for t, v in told.items():
                if t >= 0:
                    x[t] += v
        if host["mask"] is not None:
            allowed = np.unpackbits(host["mask"][r].view(np.uint8), bitorder="little")[:V]
            x[allowed == 0] = -np.inf
        out.append(x)
    return torch.from_numpy(np.stack(out))
