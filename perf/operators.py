"""The work of a paged K/V cache, as cases that can be timed and compared.

Five kinds of cases over four operators of ``paper_2311_08263_amd.PagedCache``:

  attn     attention of a batch's new rows (one token, a decoding window, a prompt chunk) over the pages (``attn``); with
           ``window`` > 0 a row sees the last ``window`` positions up to its own and the first ``sinks`` ones
  write    the K/V of new rows into the pages (``write``)
  round    the bookkeeping between two steps of a serving loop (``free``, ``fork``, ``trim``, ``grow``, ``advance``)
  fork     sequences continued from others, sharing their whole pages (``fork``)
  compact  the pages in use moved to the front of the pool (``compact``)

Where ``own`` is false, ``run`` computes the same in elementary torch operations.

A pool is [layers][pages][K/V heads][page / 32][32 * Dh], blocks of 32 positions in the library's fragment order: element
(position p, head element d) of a K block stands at ((t * 4 + s) * 16 * G + r + 16 * (d / 32)) * 8 + d % 8 with G = Dh / 32,
t = p / 4 % 2, s = d % 32 / 8, r = 4 * (p / 8) + p % 4, and of a V block at (d / 16 * 64 + d % 16 + 16 * (p / 8)) * 8 + p % 8.
``book`` holds the page table [sequences][pages a sequence], the lengths and the number of sequences that use each page.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# query heads, K/V heads, head size: Llama-2 7B / 13B / 70B, the small fp32 configuration, generic ones
HEADS = {"7b": (32, 32, 128), "13b": (40, 40, 128), "70b": (64, 8, 128), "tiny": (4, 4, 64), "g4": (16, 4, 128), "g6": (12, 2, 96),
         "mqa": (24, 1, 64), "wide": (8, 4, 256)}
EINVAL, ECAPACITY = -1, -3


def listed():
    return [
        # ------------------------------------------------ attention over pages
        # a Jacobi step of the small fp32 configuration, three short sequences: the smallest call
        {"name": "attn_tiny_f32_b3_w8", "kind": "attn", "heads": "tiny", "cache": "f32", "act": "f32", "B": 3, "lo": 60, "hi": 190, "rows": "8", "P": 32, "window": 0, "sinks": 0},
        # the benchmark's decoding step: one 7B layer, batch 1, window 16
        {"name": "attn_7b_b1_w16", "kind": "attn", "heads": "7b", "cache": "bf16", "act": "f32", "B": 1, "lo": 777, "hi": 777, "rows": "16", "P": 64, "window": 0, "sinks": 0},
        # greedy decoding of a serving batch, lengths spread over two decades: the largest K/V stream
        {"name": "attn_13b_b48_ragged", "kind": "attn", "heads": "13b", "cache": "bf16", "act": "bf16", "B": 48, "lo": 60, "hi": 8100, "rows": "1", "P": 64, "window": 0, "sinks": 0},
        # one sequence with a very long context, grouped heads: the split over the length
        {"name": "attn_70b_b1_n120k", "kind": "attn", "heads": "70b", "cache": "bf16", "act": "bf16", "B": 1, "lo": 120001, "hi": 120001, "rows": "1", "P": 256, "window": 0, "sinks": 0},
        # ------------------------------------------------ sliding window and sinks
        # streaming decoding: 16 long sequences whose pages behind the window have been given back
        {"name": "sink_7b_b16_w1", "kind": "attn", "heads": "7b", "cache": "bf16", "act": "f32", "B": 16, "lo": 9000, "hi": 20000, "rows": "1", "P": 64, "window": 2048, "sinks": 4},
        # a whole prompt under a window
        {"name": "sink_7b_p4096", "kind": "attn", "heads": "7b", "cache": "bf16", "act": "bf16", "B": 1, "lo": 0, "hi": 0, "rows": "4096", "P": 128, "window": 1024, "sinks": 4},
        # ragged prompt chunks behind long contexts, odd sizes
        {"name": "sink_70b_chunks", "kind": "attn", "heads": "70b", "cache": "bf16", "act": "f32", "B": 3, "lo": 333, "hi": 4001, "rows": "700,33,1501", "P": 128, "window": 1000, "sinks": 5},
        # ------------------------------------------------ K/V into pages
        # one new token in each of 64 sequences
        {"name": "write_70b_b64_w1", "kind": "write", "heads": "70b", "cache": "bf16", "act": "bf16", "B": 64, "lo": 100, "hi": 1999, "rows": "1", "P": 128},
        # a prompt of 4096 tokens computed in fp32, starting inside a page
        {"name": "write_7b_p4096", "kind": "write", "heads": "7b", "cache": "bf16", "act": "f32", "B": 1, "lo": 37, "hi": 37, "rows": "4096", "P": 64},
        # ------------------------------------------------ pages
        # between two steps: a quarter of the batch has ended, others are forked into its slots, windows move on
        {"name": "round_70b_b40", "kind": "round", "heads": "70b", "layers": 8, "S": 64, "B": 40, "lo": 100, "hi": 4000, "rows": "16", "P": 64, "window": 1500, "sinks": 4},
        # best of sixteen: one prompt continued fifteen times, whole 7B cache
        {"name": "fork_7b_best_of_16", "kind": "fork", "heads": "7b", "layers": 32, "S": 16, "B": 1, "lo": 1234, "hi": 1234, "children": 15, "P": 128},
        # a pool half empty after a burst, moved together so that its rear can be given back
        {"name": "compact_13b_half", "kind": "compact", "heads": "13b", "layers": 8, "S": 48, "B": 24, "lo": 50, "hi": 2000, "P": 64},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(("attn", "attn", "sink", "sink", "write", "round", "fork", "compact"))
    heads = rng.choice(sorted(HEADS))
    P = rng.choice((32, 64, 128, 256))
    if kind in ("round", "fork", "compact"):
        heads, layers = rng.choice(("7b", "13b", "70b", "g4")), rng.choice((1, 2, 4, 8))
        B = 1 + _log_int(rng, 1, 16)
        lo = _log_int(rng, 10, 500)
        c = {"kind": kind, "heads": heads, "layers": layers, "S": 2 * B + rng.randint(2, 20), "B": B, "lo": lo, "hi": lo + _log_int(rng, 10, 1500), "P": P}
        if kind == "round":
            c.update(rows=str(rng.randint(1, 40)), window=_log_int(rng, 40, 2000), sinks=rng.choice((0, 1, 4, 33)))
        if kind == "fork":
            c.update(children=rng.randint(1, 3))
        return c
    cache = "f32" if heads == "tiny" or rng.random() < 0.15 else "bf16"
    act = "f32" if cache == "f32" or rng.random() < 0.5 else "bf16"
    shape = rng.choice(("single", "window", "prompt"))
    B = _log_int(rng, 1, 64 if shape == "single" else 8)
    lo = 0 if shape == "prompt" and rng.random() < 0.4 else _log_int(rng, 1, 4000)
    hi = lo + (_log_int(rng, 1, 6000) if B > 1 or lo == 0 else 0)
    if shape == "single":
        rows = "1"
    elif shape == "window":
        rows = str(_log_int(rng, 2, 64))
    else:
        B, hi = min(B, 3), min(hi, 4000)
        rows = ",".join(str(_log_int(rng, 20, 3000)) for _ in range(B))
    c = {"kind": "write" if kind == "write" else "attn", "heads": heads, "cache": cache, "act": act, "B": B, "lo": lo, "hi": hi, "rows": rows, "P": P}
    if kind != "write":
        c.update(window=_log_int(rng, 32, 3000) if kind == "sink" else 0, sinks=rng.choice((0, 1, 4, 40)) if kind == "sink" else 0)
    return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 2e14


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= most:
            return case


# ---------------------------------------------------------------------------- sizes
def _lens(case):
    """Committed length of every sequence: spread over lo..hi evenly in their logarithm, in mixed order."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    a, b = math.log(lo + 1), math.log(hi + 1)
    lens = [int(round(math.exp(a + (b - a) * (i / max(1, B - 1)))) - 1) for i in range(B)]
    random.Random(B * 1000 + hi).shuffle(lens)
    return lens


def _rows(case):
    r = [int(x) for x in case["rows"].split(",")]
    return r if len(r) == case["B"] else [r[0]] * case["B"]


def _first_seen(n, case):
    """First position behind the sinks that the row at position n sees."""
    return max(0, n - case["window"] + 1) if case.get("window") else 0


def _pairs(n, rows, case):
    """Visible (row, position) pairs of one sequence, and positions that at least one row sees."""
    p = torch.arange(n, n + rows, dtype=torch.int64)
    lo = torch.clamp(p - case["window"] + 1, min=0) if case["window"] else torch.zeros_like(p)
    sunk = torch.minimum(lo, torch.tensor(case["sinks"] if case["window"] else 0))
    return int((p + 1 - lo + sunk).sum()), n + rows - int(lo[0]) + int(sunk[0])


def work(case):
    H, Hkv, Dh = HEADS[case["heads"]]
    if case["kind"] in ("attn", "write"):
        ca, ac = (4 if case[k] == "f32" else 2 for k in ("cache", "act"))
        lens, rows = _lens(case), _rows(case)
        if case["kind"] == "write":
            return {"bytes": sum(rows) * Hkv * Dh * 2 * (ca + ac), "flops": 0}
        pairs, seen = (sum(x) for x in zip(*(_pairs(n, r, case) for n, r in zip(lens, rows))))
        return {"bytes": seen * Hkv * Dh * 2 * ca + sum(rows) * H * (Dh * 2 * ac + 4), "flops": 4 * pairs * H * Dh}
    P, lens, layers = case["P"], _lens(case), case["layers"]
    block = 32 * Hkv * Dh * 2 * 2 * layers        # K and V of 32 positions in every layer
    book = 4 * (_table_pages(case) * case["S"] + case["S"] + _pool_pages(case))
    if case["kind"] == "compact":
        return {"bytes": 2 * book + 2 * block * (P // 32) * _moved(case), "flops": 0}
    parents = _parents(case)
    return {"bytes": 2 * book + 2 * block * sum((lens[i] % P + 31) // 32 for i in parents), "flops": 0}


def _parents(case):
    """Index among the running sequences of each new sequence's parent."""
    if case["kind"] == "fork":
        return [i for i in range(case["B"]) for _ in range(case["children"])]
    ended = case["B"] // 4
    return [ended + i % (case["B"] - ended) for i in range(ended)]


def _table_pages(case):
    rows = max(_rows(case)) if "rows" in case else 1
    return -(-(case["hi"] + 2 * rows + 1) // case["P"]) + 1


def _kept(case):
    """Page slots of every running sequence that hold something a later row sees."""
    P, out = case["P"], []
    rows = _rows(case) if case["kind"] in ("attn", "write") else [0] * case["B"]
    for n, r in zip(_lens(case), rows):
        seen = _first_seen(n, case) if case["kind"] == "attn" else 0
        out.append([i for i in range(-(-(n + r) // P)) if (i + 1) * P > seen or i * P < case.get("sinks", 0)])
    return out


def _pool_pages(case):
    used = sum(len(k) for k in _kept(case))
    if case["kind"] == "compact":
        return 2 * used + 3
    return used + 3 + used // 16 + {"fork": case["B"] * case.get("children", 0), "round": 2 * case["B"] * (2 + (max(_rows(case)) if "rows" in case else 0) // case["P"])}.get(case["kind"], 0)


def _placing(case):
    """Pages of the pool in the order in which sequences were given them: scattered."""
    ids = list(range(_pool_pages(case)))
    random.Random(case["B"] * 77 + case["hi"]).shuffle(ids)
    return ids


def _moved(case):
    used = sum(len(k) for k in _kept(case))
    return sum(i >= used for i in _placing(case)[:used])


# ---------------------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream * 7919 + 17) % (1 << 62))
    return g


def _normal(shape, seed, stream, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=_gen(seed, stream))


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def prepare(case, seed):
    H, Hkv, Dh = HEADS[case["heads"]]
    P, B, S = case["P"], case["B"], case.get("S", case["B"])
    lens, N, MP, L = _lens(case), _pool_pages(case), _table_pages(case), case.get("layers", 1)
    dtype = TYPES[case.get("cache", "bf16")]
    s = {"case": dict(case), "H": H, "Hkv": Hkv, "Dh": Dh, "P": P, "B": B, "S": S, "MP": MP, "N": N, "L": L}
    s["k"] = _normal((L, N, Hkv, P // 32, 32 * Dh), seed, 1, dtype)
    s["v"] = _normal((L, N, Hkv, P // 32, 32 * Dh), seed, 2, dtype)
    # sequences of a batch sit in slots of the table in an order of the seed's; so do their pages in the pool
    slots = random.Random(int(seed)).sample(range(S), B)
    ids = _placing(case)
    if case["kind"] != "compact":
        random.Random(int(seed) + 1).shuffle(ids)
    table, length, ref = [[-1] * MP for _ in range(S)], [0] * S, [0] * N
    for slot, n, kept in zip(slots, lens, _kept(case)):
        length[slot] = n
        for i in kept:
            table[slot][i] = ids.pop(0)
            ref[table[slot][i]] = 1
    s["book"] = _int([x for row in table for x in row] + length + ref)
    s["book0"] = s["book"].clone()
    s["seqs"] = _int(slots)
    if case["kind"] in ("attn", "write"):
        rows = _rows(case)
        s["max_rows"], n_rows = max(rows), sum(rows)
        starts = [sum(rows[:i]) for i in range(B + 1)]
        s["row_start"] = _int(starts)
        s["row_b"] = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(rows, device="cuda"))
        s["row_j"] = torch.arange(n_rows, device="cuda") - s["row_start"].long()[s["row_b"]]
        s["T"] = -(-(max(n + r for n, r in zip(lens, rows))) // P)
        s["ragged"] = len(set(rows)) > 1
        act = TYPES[case["act"]]
        if case["kind"] == "attn":
            s["q"] = _normal((n_rows, H, Dh), seed, 3, act, 1.5)
        else:
            s["new_k"], s["new_v"] = _normal((n_rows, Hkv, Dh), seed, 4, act), _normal((n_rows, Hkv, Dh), seed, 5, act)
    else:
        free = [x for x in range(S) if x not in slots]
        parents = [slots[i] for i in _parents(case)]
        if case["kind"] == "round":
            s["ended"] = _int(slots[:len(parents)])
            s["src"], s["dst"] = _int(parents), _int(slots[:len(parents)])
            s["rows"] = torch.full((B,), int(case["rows"]), dtype=torch.int32, device="cuda")
            s["accepted"] = torch.randint(1, int(case["rows"]) + 1, (B,), generator=_gen(seed, 6), dtype=torch.int32, device="cuda")
        elif case["kind"] == "fork":
            s["src"], s["dst"] = _int(parents), _int(free[:len(parents)])
    if own:
        from paper_2311_08263_amd import PagedCache
        s["cache"] = PagedCache(N, P, Hkv, Dh, dtype=dtype, n_layers=L, max_seqs=S, max_pages=MP, k=s["k"], v=s["v"], book=s["book"])
    torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------------------- the calls
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    c, case = s["cache"], s["case"]
    where = dict(seqs=s["seqs"])
    if case["kind"] in ("attn", "write") and s["ragged"]:
        where.update(row_start=s["row_start"], max_rows=s["max_rows"])
    if case["kind"] == "attn":
        out, lse = c.attn(s["q"], window=case["window"], sinks=case["sinks"], want_lse=True, **where)
        return {"out": out, "lse": lse}
    if case["kind"] == "write":
        c.write(s["new_k"], s["new_v"], **where)
        return {"k": s["k"], "v": s["v"]}
    s["book"].copy_(s["book0"])
    if case["kind"] == "compact":
        used = c.compact()
        return {"book": s["book"], "used": used, "k": s["k"], "v": s["v"]}
    if case["kind"] == "fork":
        return {"status": c.fork(s["src"], s["dst"]), "book": s["book"], "k": s["k"], "v": s["v"]}
    done = [c.free(s["ended"]), c.fork(s["src"], s["dst"]), c.trim(s["seqs"], case["window"], case["sinks"]), c.grow(s["seqs"], s["rows"]),
            c.advance(s["seqs"], s["accepted"])]
    return {"status": done, "book": s["book"], "k": s["k"], "v": s["v"]}


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "attn":
        return _plain_attn(s)
    if case["kind"] == "write":
        return _plain_write(s)
    s["book"].copy_(s["book0"])
    if case["kind"] == "compact":
        return {"used": _plain_compact(s), "book": s["book"], "k": s["k"], "v": s["v"]}
    if case["kind"] == "fork":
        return {"status": _plain_fork(s), "book": s["book"], "k": s["k"], "v": s["v"]}
    done = [_plain_free(s), _plain_fork(s), _plain_trim(s), _plain_grow(s), _plain_advance(s)]
    return {"status": done, "book": s["book"], "k": s["k"], "v": s["v"]}


def _books(s):
    """Views of the table, the lengths and the use counts inside the book."""
    S, MP = s["S"], s["MP"]
    return s["book"][:S * MP].view(S, MP), s["book"][S * MP:S * MP + S], s["book"][S * MP + S:]


def _plain_attn(s):
    H, Hkv, Dh, P, T, R = s["H"], s["Hkv"], s["Dh"], s["P"], s["T"], s["max_rows"]
    window, sinks, B, G = s["case"]["window"], s["case"]["sinks"], s["B"], Dh // 32
    table, length, _ = _books(s)
    seqs = s["seqs"].long()
    pages = table[seqs, :T]
    at = pages.clamp(min=0).long()
    # [B][pages][Hkv][blocks] and the places inside a block in the order position, head element
    k = s["k"][0][at].float().view(B, T, Hkv, P // 32, 2, 4, G, 4, 4, 8).permute(0, 2, 1, 3, 7, 4, 8, 6, 5, 9).reshape(B, Hkv, T * P, Dh)
    v = s["v"][0][at].float().view(B, T, Hkv, P // 32, Dh // 16, 4, 16, 8).permute(0, 2, 1, 3, 5, 7, 4, 6).reshape(B, Hkv, T * P, Dh)
    rows = (s["row_start"][:B, None].long() + torch.arange(R, device="cuda")).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[rows].view(B, R, Hkv, H // Hkv, Dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, Dh)
    scores = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(Dh)
    pos = torch.arange(T * P, device="cuda")
    here = length[seqs].long()[:, None, None] + torch.arange(R, device="cuda")[:, None]
    seen = (pos <= here) & (pages >= 0).repeat_interleave(P, 1)[:, None]
    if window:
        seen &= (pos > here - window) | (pos < sinks)
    scores = scores.view(B, Hkv, R, H // Hkv, -1).masked_fill_(~seen[:, None, :, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    scores = scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, Hkv, -1, T * P), v).view(B, Hkv, R, H // Hkv, Dh) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.permute(0, 2, 1, 3, 4).reshape(B, R, H * Dh)[s["row_b"], s["row_j"]]
    lse = (top + total.log()).permute(0, 2, 1, 3, 4).reshape(B, R, H)[s["row_b"], s["row_j"]]
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _plain_write(s):
    Hkv, Dh, P = s["Hkv"], s["Dh"], s["P"]
    G, PB, N = Dh // 32, P // 32, s["N"]
    table, length, _ = _books(s)
    seq = s["seqs"].long()[s["row_b"]]
    pos = length[seq].long() + s["row_j"]
    page, b, p = table[seq, pos // P].long(), pos % P // 32, pos % 32
    k, v = s["new_k"].to(s["k"].dtype).view(-1, Hkv, G, 4, 8), s["new_v"].to(s["v"].dtype).view(-1, Hkv, Dh // 16, 16)
    s["k"][0].view(N, Hkv, PB, 2, 4, G, 4, 4, 8)[page, :, b, p // 4 % 2, :, :, p // 8, p % 4] = k.transpose(2, 3)
    s["v"][0].view(N, Hkv, PB, Dh // 16, 4, 16, 8)[page, :, b, :, p // 8, :, p % 8] = v
    return {"k": s["k"], "v": s["v"]}


def _repeated(x):
    """Entries whose value an earlier entry has."""
    i = torch.arange(x.numel(), device="cuda")
    return ((x[:, None] == x[None]) & (i[None] < i[:, None])).any(1)


def _with_row(x):
    """One more row than `x` has, for what is written nowhere."""
    return torch.cat([x, x[:1]])


def _plain_fork(s):
    table, length, ref = _books(s)
    S, P, N, src, dst = s["S"], s["P"], s["N"], s["src"].long(), s["dst"].long()
    a, b = src.clamp(0, S - 1), dst.clamp(0, S - 1)
    ok = (src == a) & (dst == b) & (length[b] == 0) & (table[b, 0] < 0) & ~_repeated(dst) & ~(src[:, None] == dst[None]).any(1)
    n = length[a].long()
    last, part = n // P, n % P
    slots = torch.arange(s["MP"], device="cuda")
    old = table[a, last.clamp(max=s["MP"] - 1)].long()
    need = ok & (part > 0) & (old >= 0)
    before = need.long().cumsum(0)
    given = need & (before <= (ref == 0).sum())
    short = need & ~given
    ok = ok & ~short
    page = torch.sort((ref != 0).int(), stable=True).indices[(before - 1).clamp(0, N - 1)]     # the lowest free ones, in order
    child = torch.where(slots < last[:, None], table[a], -1)
    child = torch.where(given[:, None] & (slots == last[:, None]), page[:, None].int(), child)
    to = torch.where(ok, b, S)
    uses = _with_row(ref).index_put_((torch.where(ok[:, None] & (child >= 0), child, N).long(),), torch.ones_like(child), accumulate=True)
    table.copy_(_with_row(table).index_copy_(0, to, child)[:S])
    length.copy_(_with_row(length).index_copy_(0, to, n.int())[:S])
    ref.copy_(uses[:N])
    x, y = old[given], page[given]
    held = (torch.arange(P // 32, device="cuda") < ((part[given] + 31) // 32)[:, None])[None, :, None, :, None]
    for pool in (s["k"], s["v"]):
        pool[:, y] = torch.where(held, pool[:, x], pool[:, y])
    return torch.where(ok, 0, torch.where(short, ECAPACITY, EINVAL)).int()


def _release(s, seqs, leave):
    """The pages of table entries [entries][slots] that leave their sequences; an entry that is named twice leaves once."""
    table, _, ref = _books(s)
    S, MP, N = s["S"], s["MP"], s["N"]
    flag = torch.zeros(S + 1, MP, dtype=torch.bool, device="cuda")
    flag.index_put_((torch.where((seqs >= 0) & (seqs < S), seqs, S),), leave, accumulate=True)
    gone = flag[:S] & (table >= 0)
    uses = _with_row(ref).index_put_((torch.where(gone, table, N).long(),), torch.full_like(table, -1), accumulate=True)
    ref.copy_(uses[:N])
    table.masked_fill_(gone, -1)


def _plain_free(s):
    seqs = s["ended"].long()
    _, length, _ = _books(s)
    inside = (seqs >= 0) & (seqs < s["S"])
    _release(s, seqs, inside[:, None].expand(-1, s["MP"]))
    length.copy_(_with_row(length).index_fill_(0, torch.where(inside, seqs, s["S"]), 0)[:s["S"]])
    return torch.where(inside, 0, EINVAL).int()


def _plain_trim(s):
    seqs, P = s["seqs"].long(), s["P"]
    _, length, _ = _books(s)
    inside = (seqs >= 0) & (seqs < s["S"])
    n = length[seqs.clamp(0, s["S"] - 1)].long()
    first = torch.arange(s["MP"], device="cuda") * P
    _release(s, seqs, inside[:, None] & (first >= s["case"]["sinks"]) & (first + P - 1 <= n[:, None] - s["case"]["window"]))
    return torch.where(inside, 0, EINVAL).int()


def _plain_grow(s):
    table, length, ref = _books(s)
    S, P, N, seqs, rows = s["S"], s["P"], s["N"], s["seqs"].long(), s["rows"].long()
    a = seqs.clamp(0, S - 1)
    n = length[a].long()
    end = (n + rows + P - 1) // P
    valid = (seqs == a) & (rows >= 0) & ~_repeated(seqs)
    large = valid & (end > s["MP"])
    valid = valid & ~large
    slots = torch.arange(s["MP"], device="cuda")
    want = valid[:, None] & (slots >= (n // P)[:, None]) & (slots < end[:, None]) & (table[a] < 0)
    before = want.sum(1).cumsum(0)
    short = valid & want.any(1) & (before > (ref == 0).sum())
    take = want & ~short[:, None]
    rank = want.view(-1).long().cumsum(0).view(want.shape) - 1
    page = torch.sort((ref != 0).int(), stable=True).indices[rank.clamp(0, N - 1)]
    new = torch.where(take, page.int(), table[a])
    table.copy_(_with_row(table).index_copy_(0, torch.where(valid, a, S), new)[:S])
    ref.copy_(_with_row(ref).index_fill_(0, torch.where(take, page, N).view(-1), 1)[:N])
    return torch.where(valid & ~short, 0, torch.where(large | short, ECAPACITY, EINVAL)).int()


def _plain_advance(s):
    table, length, _ = _books(s)
    S, P, seqs, rows = s["S"], s["P"], s["seqs"].long(), s["accepted"].long()
    a = seqs.clamp(0, S - 1)
    n = length[a].long()
    end = (n + rows + P - 1) // P
    slots = torch.arange(s["MP"], device="cuda")
    valid = (seqs == a) & (rows >= 0) & ~_repeated(seqs)
    missing = (end > s["MP"]) | ((slots >= (n // P)[:, None]) & (slots < end[:, None]) & (table[a] < 0)).any(1)
    ok = valid & ~missing
    length.copy_(_with_row(length).index_copy_(0, torch.where(ok, a, S), (n + rows).int())[:S])
    return torch.where(ok, 0, torch.where(valid, ECAPACITY, EINVAL)).int()


def _plain_compact(s):
    table, _, ref = _books(s)
    N = s["N"]
    inuse, ids = ref > 0, torch.arange(N, device="cuda")
    used = inuse.sum()
    src, dst = (inuse & (ids >= used)).nonzero()[:, 0], (~inuse & (ids < used)).nonzero()[:, 0]
    to = _with_row(ids).index_copy_(0, src, dst).int()
    to[N] = -1
    table.copy_(to[torch.where(table >= 0, table, N).long()])
    ref[dst] = ref[src]
    ref[src] = 0
    for pool in (s["k"], s["v"]):
        pool[:, dst] = pool[:, src]
    return used.int()


# ---------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    if case["kind"] not in ("attn", "write"):
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    H, Hkv, Dh = HEADS[case["heads"]]
    P, S, MP = case["P"], case.get("S", case["B"]), s["MP"]
    book = s["book"].tolist()
    slots, starts, rows = s["seqs"].tolist(), s["row_start"].tolist(), _rows(case)
    dh, G = torch.arange(Dh, device="cuda"), Dh // 32

    def places(slot, pos):
        """Page and offsets of K and V elements [positions][Dh] inside a page's block of one head."""
        page = torch.tensor(book[slot * MP:(slot + 1) * MP], device="cuda")[pos // P]
        p, at = pos[:, None] % 32, (pos[:, None] % P // 32) * 32 * Dh
        r = 4 * (p // 8) + p % 4
        ke = at + ((p // 4 % 2 * 4 + dh % 32 // 8) * 16 * G + r + 16 * (dh // 32)) * 8 + dh % 8
        ve = at + (dh // 16 * 64 + dh % 16 + 16 * (p // 8)) * 8 + p % 8
        return page, ke, ve

    if case["kind"] == "write":
        k, v = s["k"].double().view(s["N"], Hkv, -1), s["v"].double().view(s["N"], Hkv, -1)
        for slot, a, r in zip(slots, starts, rows):
            pos = book[S * MP + slot] + torch.arange(r, device="cuda")
            page, ke, ve = places(slot, pos)
            for h in range(Hkv):
                k[page[:, None], h, ke] = s["new_k"][a:a + r, h].double()
                v[page[:, None], h, ve] = s["new_v"][a:a + r, h].double()
        return {"k": k.view(s["k"].shape), "v": v.view(s["v"].shape)}
    out = torch.zeros(sum(rows), H * Dh, dtype=torch.float64, device="cuda")
    lse = torch.zeros(sum(rows), H, dtype=torch.float64, device="cuda")
    for slot, a, r in zip(slots, starts, rows):
        n = book[S * MP + slot]
        j = torch.arange(n, n + r, device="cuda")
        first, sunk = _first_seen(n, case), min(case["sinks"], _first_seen(n, case))
        pos = torch.cat([torch.arange(sunk, device="cuda"), torch.arange(first, n + r, device="cuda")])
        page, ke, ve = places(slot, pos)
        hidden = pos > j[:, None]
        if case["window"]:
            hidden |= (pos <= j[:, None] - case["window"]) & (pos >= case["sinks"])
        for h in range(H):
            g = h // (H // Hkv)
            k, v = (pool[0, :, g].reshape(s["N"], -1)[page[:, None], e].double() for pool, e in ((s["k"], ke), (s["v"], ve)))
            score = (s["q"][a:a + r, h].double() @ k.t() * Dh ** -0.5).masked_fill(hidden, -math.inf)
            lse[a:a + r, h] = torch.logsumexp(score, 1)
            out[a:a + r, h * Dh:(h + 1) * Dh] = torch.softmax(score, 1) @ v
    return {"out": out, "lse": lse}
