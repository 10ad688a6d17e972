"""The K/V cache in pages on the GPU against the same in plain Python (paged_util): attention in 64 bits, whole numbers and moved values bit for bit.

Tolerances.  fp32 rows: queries and weights keep 24 bits, products are exact, sums run in fp32 (pieces of at most 32 terms per
block): a relative error of a few 2^-24 of the scores' size (below 8 here) in every weight, 2e-6 of the norm as in the tests of the other attention
kernels.  bf16 rows: the rounding of the output, half a step of 2^-7 relative to each value, and weights in two parts (2^-17)."""
import random

import pytest

from gpu_util import say
from paged_util import Plain, canonical

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fc():
    import paper_2311_08263_amd as m
    return m


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rel(a, b):
    import torch
    a, b = a.double(), b.double()
    return float(torch.linalg.norm(a - b) / torch.linalg.norm(b))


def make(fc, lens, rows, P, Hkv, Dh, cache="bf16", layers=1, spare=3, fill=float("nan"), window=0, sinks=0, seed=0):
    """A cache with sequences of these lengths in scattered slots and pages, and room for `rows` more positions of each; positions that
    nobody has written hold `fill`.  Returns it with the slots."""
    import torch
    dt = torch.bfloat16 if cache == "bf16" else torch.float32
    B = len(lens)
    S, MP = B + 2, max(-(-(n + r) // P) for n, r in zip(lens, rows)) + 1
    N = sum(-(-(n + r) // P) for n, r in zip(lens, rows)) + spare
    c = fc.PagedCache(N, P, Hkv, Dh, dtype=dt, n_layers=layers, max_seqs=S, max_pages=MP)
    rnd = random.Random(seed)
    slots, pages = rnd.sample(range(S), B), rnd.sample(range(N), N)
    table, ref = [[-1] * MP for _ in range(S)], [0] * N
    ln = [0] * S
    for s, n, r in zip(slots, lens, rows):
        ln[s] = n
        for i in range(-(-(n + r) // P)):
            table[s][i] = pages.pop()
            ref[table[s][i]] = 1
    c.book.copy_(ints([x for row in table for x in row] + ln + ref))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for pool in (c.k, c.v):
        pool.copy_(torch.randn(pool.shape, generator=g, device="cuda"))
    if fill is not None:
        for pool, which in ((c.k, 0), (c.v, 1)):
            order = canonical(torch.arange(32 * Dh, device="cuda").view(1, 1, 1, 1, -1), Dh)[which].reshape(32, Dh)
            used = torch.zeros(N, P, dtype=torch.bool)
            for s, n, r in zip(slots, lens, rows):
                for p in range(n + r):
                    used[table[s][p // P], p % P] = True
            for page, pos in (~used).nonzero().tolist():
                pool[:, page, :, pos // 32, order[pos % 32]] = fill
    return c, slots


def queries(rows, H, Dh, act, seed=5):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (1.5 * torch.randn(sum(rows), H, Dh, generator=g, device="cuda")).to(torch.bfloat16 if act == "bf16" else torch.float32)


def starts(rows):
    return ints([sum(rows[:i]) for i in range(len(rows) + 1)])


def check(out, lse, want, act):
    import torch
    o, l = want
    seen = torch.isfinite(l)
    assert torch.equal(torch.isneginf(lse), ~seen)
    assert rel(out, o) < (2e-6 if act == "f32" else 2 ** -8 + 2 ** -16)
    assert float((lse.double() - l)[seen].abs().max()) < 1e-5          # 2^-24 of scores and logs below 16, a few times


CASES = [
    # lens, rows, P, H, Hkv, Dh, cache, act, window, sinks
    ([0], [1], 32, 1, 1, 32, "bf16", "f32", 0, 0),
    ([0, 31, 32, 33, 200], [1] * 5, 32, 4, 4, 128, "bf16", "f32", 0, 0),
    ([0, 31, 32, 33, 200], [1] * 5, 64, 8, 2, 128, "bf16", "bf16", 0, 0),
    ([5, 77, 300], [8, 8, 8], 32, 4, 4, 64, "f32", "f32", 0, 0),
    ([5, 77, 300], [3, 1, 16], 128, 12, 2, 96, "bf16", "f32", 0, 0),
    ([0, 63, 130], [17, 5, 33], 64, 6, 2, 192, "bf16", "bf16", 0, 0),
    ([9, 130], [11, 40], 32, 4, 1, 256, "f32", "f32", 0, 0),
    ([9, 130], [11, 40], 64, 4, 2, 256, "bf16", "f32", 0, 0),
    ([700], [1], 256, 64, 1, 64, "bf16", "bf16", 0, 0),                    # 64 heads on one
    ([1, 400], [70, 1], 32, 3, 3, 32, "f32", "f32", 0, 0),
    ([0], [150], 64, 4, 2, 128, "bf16", "f32", 0, 0),                      # a prompt from its start
    ([100, 0], [0, 9], 32, 2, 2, 128, "bf16", "f32", 0, 0),                # a sequence without rows
    # windows
    ([0, 31, 32, 33, 200, 300], [1] * 6, 32, 4, 2, 128, "bf16", "f32", 1, 0),
    ([0, 31, 32, 33, 200, 300], [1] * 6, 32, 4, 2, 128, "bf16", "bf16", 33, 4),
    ([40, 200, 333], [7, 40, 1], 32, 4, 2, 128, "bf16", "f32", 64, 33),
    ([40, 200, 333], [7, 40, 1], 64, 4, 4, 64, "f32", "f32", 50, 4),
    ([0], [300], 32, 4, 2, 128, "bf16", "bf16", 70, 5),
    ([0], [300], 64, 2, 2, 128, "bf16", "f32", 1, 1),
    ([10], [30], 32, 2, 1, 96, "bf16", "f32", 10 ** 9, 10 ** 9),
    ([500], [2], 32, 4, 1, 128, "bf16", "f32", 40, 100),
    # 17 to 32 rows of a K/V head
    ([9, 700], [9, 14], 32, 4, 2, 64, "bf16", "f32", 0, 0),
    ([9, 700], [9, 14], 32, 4, 2, 64, "bf16", "bf16", 90, 2),
    ([9, 700], [9, 14], 32, 4, 2, 64, "f32", "f32", 0, 0),
    ([31, 400], [5, 8], 64, 4, 1, 96, "bf16", "f32", 0, 0),
    ([31, 400], [5, 8], 64, 4, 1, 96, "f32", "f32", 33, 1),
    ([31, 1400], [17, 31], 64, 2, 2, 128, "bf16", "bf16", 0, 0),
    ([31, 400], [17, 31], 64, 2, 2, 128, "f32", "f32", 0, 0),
    ([31, 400], [17, 31], 64, 1, 1, 192, "f32", "f32", 0, 0),
    ([31, 400], [5, 8], 64, 4, 1, 256, "bf16", "bf16", 0, 0),
    ([31, 400], [5, 8], 64, 4, 1, 192, "bf16", "f32", 50, 3),
]


@pytest.mark.parametrize("lens,rows,P,H,Hkv,Dh,cache,act,window,sinks", CASES)
def test_attention(fc, lens, rows, P, H, Hkv, Dh, cache, act, window, sinks):
    say(f"paged attention {lens} {rows} P={P} H={H}/{Hkv} Dh={Dh} {cache} {act} window={window} sinks={sinks}")
    c, slots = make(fc, lens, rows, P, Hkv, Dh, cache)
    q = queries(rows, H, Dh, act)
    out, lse = c.attn(q, seqs=ints(slots), row_start=starts(rows), max_rows=max(rows), window=window, sinks=sinks, want_lse=True)
    check(out, lse, Plain(c).attn(Dh, 0, slots, rows, q, window, sinks), act)
    if len(set(rows)) == 1:                  # the dense form of the call: the same bits
        assert (out == c.attn(q, seqs=ints(slots), window=window, sinks=sinks)).all()


@pytest.mark.parametrize("H,Hkv,rows,window,sinks", [(4, 4, [6, 1, 9], 0, 0), (4, 4, [6, 1, 20], 0, 0), (8, 2, [16, 9, 3], 45, 3), (2, 1, [100, 7, 70], 0, 0)])
@pytest.mark.parametrize("cache,act", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
def test_attention_takes_nothing_from_hidden_positions(fc, H, Hkv, rows, window, sinks, cache, act):
    """V holds an infinity and a NaN where only some of a unit's rows see them, and NaN wherever nobody has written; pages are missing in the
    middle, one sequence number is out of range, and the rows of none stay as they were."""
    import torch
    say(f"paged attention, hidden positions H={H}/{Hkv} {rows} window={window} {cache} {act}")
    lens, P, Dh = [70, 200, 33], 32, 128
    c, slots = make(fc, lens, rows, P, Hkv, Dh, cache)
    c.table[slots[1], 3] = -1
    c.table[slots[1], 4] = c._desc.n_pages + 5
    q = queries(rows + [4], H, Dh, act)
    plain = Plain(c)
    plain.table[slots[1]][4] = -1
    seqs, all_rows = slots + [99], rows + [2]                      # two rows of no sequence, two behind the last
    want, wlse = plain.attn(Dh, 0, seqs, all_rows, q, window, sinks)
    # position lens[0] + 1 of the first sequence: seen from its second row on
    p = lens[0] + 1
    order = canonical(torch.arange(32 * Dh, device="cuda").view(1, 1, 1, 1, -1), Dh)[1].reshape(32, Dh)
    page = c.table[slots[0], p // P]
    c.v[0, page, :, 0, order[p % 32, 37]], c.v[0, page, :, 0, order[p % 32, 90]] = float("inf"), float("nan")
    out = torch.full((sum(rows) + 4, H * Dh), 7.0, dtype=q.dtype, device="cuda")
    _, lse = c.attn(q, seqs=ints(seqs), row_start=starts(all_rows), max_rows=max(rows), window=window, sinks=sinks, out=out, want_lse=True)
    assert (out[-2:] == 7).all() and (out[-4:-2] == 0).all()
    o = out.view(-1, H, Dh)[1:rows[0]]
    assert torch.isinf(o[..., 37]).all() and torch.isnan(o[..., 90]).all()
    o[..., 37], o[..., 90] = want.view(-1, H, Dh)[1:rows[0], :, 37].to(q.dtype), want.view(-1, H, Dh)[1:rows[0], :, 90].to(q.dtype)
    check(out[:-2], lse[:-2], (want[:-2], wlse[:-2]), act)


@pytest.mark.parametrize("rows", [3, 80])
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_attention_at_the_ends_of_the_range(fc, rows, act):
    """Queries up to the largest numbers, and rows all of whose scores lie far below zero or far above."""
    import torch
    say(f"paged attention at the ends of the range rows={rows} {act}")
    c, slots = make(fc, [90], [rows], 32, 2, 128)
    q = queries([rows], 4, 128, "f32")
    for scale_q, scale_k in ((3e38 / 1.5, 1e-30), (1e18, -1e15), (1e18, 1e15)):
        qq = (torch.sign(q) * scale_q if scale_q > 1e30 else q.abs() * scale_q).to(torch.float32 if act == "f32" else torch.bfloat16)
        c2, _ = make(fc, [90], [rows], 32, 2, 128)
        c2.k.copy_((c.k.float() * scale_k if scale_q > 1e30 else c.k.float().abs() * scale_k).bfloat16())
        out, lse = c2.attn(qq, seqs=ints(slots), want_lse=True)
        want, wl = dense(c2, slots, [rows], qq, 0, 0)
        assert rel(out, want) < (2e-6 if act == "f32" else 2 ** -8 + 2 ** -16) and rel(lse, wl) < 2e-6


def test_one_sequence_twice(fc):
    """Two passes of a sequence in one call (drafts that share its pages): each gets its own result."""
    import torch
    say("paged attention, a sequence twice")
    c, slots = make(fc, [300, 40], [2, 2], 32, 2, 128)
    q = queries([6], 4, 128, "f32")
    out = c.attn(q, seqs=ints([slots[0], slots[1], slots[0]]))
    assert torch.equal(out[:2], c.attn(q[:2].contiguous(), seqs=ints(slots[:1]))) and rel(out, Plain(c).attn(128, 0, [slots[0], slots[1], slots[0]], [2, 2, 2], q, 0, 0)[0]) < 2e-6


def test_pools_of_more_than_four_gigabytes(fc):
    """Pages behind the 32-bit offsets of bytes and of values: written, read by both kernels, shared, copied and moved."""
    import torch
    say("paged cache of 2 x 9.8 GB")
    N, P, Dh = 300000, 32, 256
    c = fc.PagedCache(N, P, 2, Dh, max_seqs=3, max_pages=8)
    c.ref[:N - 9] = 1                                  # all but the last nine pages are taken
    rows = [100, 100]
    seqs = ints([2, 0])
    assert c.grow(seqs, ints(rows)).tolist() == [0, 0] and int(c.table[c.table >= 0].min()) == N - 9
    k, v, q = (queries(rows, 2, Dh, "bf16", i) for i in (1, 2, 3))
    c.write(k, v, seqs=seqs)
    assert c.advance(seqs, ints([50, 50])).tolist() == [0, 0]

    def check_rows(slot, a):
        pages = c.table[slot, :4].long()
        for pool, x, which in ((c.k, k, 0), (c.v, v, 1)):
            assert torch.equal(canonical(pool[:, pages], Dh)[which][0].transpose(1, 2).reshape(-1, 2, Dh)[:100], x[a:a + 100])
        for n in (1, 40):                              # one row and many, each at a position that has been written
            out = c.attn(q[a:a + n], seqs=ints([slot])).view(n, 2, Dh)
            hidden = torch.arange(50 + n, device="cuda") > torch.arange(50, 50 + n, device="cuda")[:, None]
            for h in (0, 1):
                score = (q[a:a + n, h].double() @ k[a:a + 50 + n, h].double().T / Dh ** 0.5).masked_fill(hidden, -torch.inf)
                assert rel(out[:, h], torch.softmax(score, 1) @ v[a:a + 50 + n, h].double()) < 2 ** -8 + 2 ** -16
    check_rows(2, 0)
    check_rows(0, 100)
    assert c.fork(ints([2]), ints([1])).tolist() == [0] and int(c.table[1, 1]) == N - 1 and int(c.table[1, 0]) == int(c.table[2, 0])
    one, two = canonical(c.k[:, [int(c.table[2, 1]), N - 1]], Dh)[0][0]
    assert torch.equal(one[:, :18], two[:, :18])
    c.ref[:N - 9] = 0
    used = int(c.compact())
    assert used == 9 and int(c.table.max()) == 8 and int(c.ref[:9].min()) >= 1 and int(c.ref[9:].max()) == 0
    check_rows(2, 0)


def test_refusals_of_the_binding(fc):
    """What the binding refuses before the library sees it."""
    import torch
    say("paged cache, refusals of the binding")
    c, slots = make(fc, [40, 7], [5, 5], 64, 2, 128)
    s, q = ints(slots), queries([10], 4, 128, "f32")
    k = queries([10], 2, 128, "f32")

    def refused(call, text):
        with pytest.raises(fc.FastcotError, match=text) as e:
            call()
        assert e.value.rc == -1
    refused(lambda: c.grow(s.cpu(), s), "seqs")
    refused(lambda: c.grow(s.long(), s), "seqs")
    refused(lambda: c.grow(s, s[:1]), "rows")
    refused(lambda: c.fork(s, ints([1, 2, 3])), "dst")
    refused(lambda: c.trim(s[None], 5), "seqs")
    refused(lambda: c.free(ints([0, 1, 2, 3])[::2]), "seqs")
    refused(lambda: c.trim(s, 0), "window")
    refused(lambda: c.attn(q[:9], seqs=s), "row_start")
    refused(lambda: c.attn(q.cpu(), seqs=s), "q:")
    refused(lambda: c.attn(q.half(), seqs=s), "q:")
    refused(lambda: c.attn(q[..., :64], seqs=s), "q:")
    refused(lambda: c.attn(q.transpose(1, 2).contiguous().transpose(1, 2), seqs=s), "q:")
    refused(lambda: c.attn(queries([10], 3, 128, "f32"), seqs=s), "heads")
    refused(lambda: c.attn(q, seqs=s, out=torch.empty(10, 512, dtype=torch.bfloat16, device="cuda")), "out")
    refused(lambda: c.attn(q, seqs=s, scratch=c.scratch[:256]), "scratch")
    refused(lambda: c.attn(q, seqs=s, row_start=ints([0, 10])), "row_start")
    refused(lambda: c.attn(q, layer=1, seqs=s), "layer")
    refused(lambda: c.write(k, k.bfloat16(), seqs=s), "differ")
    refused(lambda: c.write(k, k[:8], seqs=s), "differ")
    refused(lambda: c.write(q[:, ::2], q[:, ::2], seqs=s), "follow")
    refused(lambda: c.write(k, torch.cat([k, k], 1)[:, :2], seqs=s), "strides")
    for bad in (dict(page_size=48), dict(head_dim=80), dict(dtype=torch.float16), dict(book=torch.zeros(5, dtype=torch.int32, device="cuda")),
                dict(k=torch.zeros(1, 10, 2, 2, 4096, device="cuda"))):
        refused(lambda: fc.PagedCache(**{**dict(n_pages=10, page_size=64, n_kv_heads=2, head_dim=128), **bad}), None)
    assert c.attn(q[:0], seqs=s[:0]).shape == (0, 512) and c.grow(s[:0], s[:0]).numel() == 0


def test_on_another_stream(fc):
    """The calls go to the stream that is current, and wait for nobody else's."""
    import torch
    say("paged cache on another stream")
    c, slots = make(fc, [100], [3], 32, 2, 128)
    q, s = queries([3], 4, 128, "f32"), ints(slots)
    want = c.attn(q, seqs=s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(20):
            big = big @ big * 1e-4
        qq = q * (big[0, 0] * 0 + 1)                   # ready only when the side stream has come here
        out = c.attn(qq, seqs=s)
    side.synchronize()
    assert torch.equal(out, want)


def test_attention_strides(fc):
    """Queries as part of a wider matrix, heads at a stride of their own, an output among others, another layer."""
    import torch
    say("paged attention, strides")
    c, slots = make(fc, [40, 7], [5, 5], 64, 2, 128, layers=3)
    wide = queries([10], 12, 128, "f32")
    q = wide[:, 2:10:2]
    out = torch.zeros(10, 1024, device="cuda")
    c.attn(q, layer=2, seqs=ints(slots), out=out[:, 256:768])
    want = Plain(c).attn(128, 2, slots, [5, 5], q, 0, 0)[0]
    assert rel(out[:, 256:768], want) < 2e-6 and (out[:, :256] == 0).all() and (out[:, 768:] == 0).all()


@pytest.mark.parametrize("lens,rows,P,Hkv,Dh,cache,act", [
    ([0, 31, 40], [1, 1, 1], 32, 2, 128, "bf16", "bf16"), ([5, 64], [70, 3], 64, 1, 96, "bf16", "f32"), ([1, 30], [7, 8], 32, 4, 64, "f32", "f32"),
    ([0], [200], 128, 2, 256, "bf16", "f32"), ([3], [129], 32, 1, 32, "bf16", "bf16"), ([8, 16], [24, 40], 32, 3, 192, "f32", "f32"),
    ([31, 2], [2, 40], 64, 2, 256, "f32", "f32")])
def test_write(fc, lens, rows, P, Hkv, Dh, cache, act):
    """Rows at any offset inside a page; values that fp32 rounds up and down; a row without a page is dropped, nothing else changes."""
    import torch
    say(f"paged write {lens} {rows} P={P} Hkv={Hkv} Dh={Dh} {cache} {act}")
    c, slots = make(fc, lens, rows, P, Hkv, Dh, cache, layers=2)
    c.table[slots[-1], (lens[-1] + rows[-1] - 1) // P] = -1
    k, v = queries(rows, Hkv, Dh, act, 1), queries(rows, 2 * Hkv, Dh, act, 2)[:, Hkv:]
    k = torch.cat([k, k], 1)[:, :Hkv]                      # a row stride that is not the row
    plain = Plain(c)
    c.write(k, v, layer=1, seqs=ints(slots), row_start=starts(rows), max_rows=max(rows))
    plain.write(Dh, 1, slots, rows, k, v)
    bits = torch.int16 if cache == "bf16" else torch.int32
    assert torch.equal(c.k.view(bits), plain.k.view(bits)) and torch.equal(c.v.view(bits), plain.v.view(bits))


def same_status(got, want):
    assert got.tolist() == want


def test_grow_and_advance(fc):
    say("paged grow and advance")
    c = fc.PagedCache(9, 32, 1, 32, max_seqs=5, max_pages=4)
    c.k.zero_(), c.v.zero_()
    plain = Plain(c)
    for seqs, rows in (([3, 0, 3, 9, -1, 2], [33, 1, 1, 1, 1, -5]), ([1, 3], [0, 95]), ([0, 1, 2], [40, 129, 128]), ([4, 2, 0, 1], [64, 1, 33, 1]), ([2], [2 ** 31 - 1])):
        seqs, rows = seqs[:5], rows[:5]
        same_status(c.grow(ints(seqs), ints(rows)), plain.grow(seqs, rows))
        plain.same(c)
        rows = [r // 2 for r in rows]
        same_status(c.advance(ints(seqs), ints(rows)), plain.advance(seqs, rows))
        plain.same(c)


def test_fork_trim_free_compact(fc):
    """Forks that are refused (occupied, twice, a source that is being filled, out of range, no page left), pages that several sequences share and leave one
    by one, windows and sinks that end inside a page, entries named twice."""
    say("paged fork, trim, free, compact")
    for P, cache in ((32, "f32"), (128, "bf16")):
        lens = [3 * P + 5, 2 * P, 1, P + 40, 0]
        c, slots = make(fc, lens, [0] * 5, P, 2, 64, cache, layers=2, spare=3, fill=None)
        plain = Plain(c)
        others = [s for s in range(7) if s not in slots]
        a, b = others
        same_status(c.fork(ints([slots[0], slots[0], slots[1], 7, slots[3]]), ints([a, a, slots[2], b, -1])), plain.fork([slots[0], slots[0], slots[1], 7, slots[3]], [a, a, slots[2], b, -1]))
        plain.same(c)
        same_status(c.fork(ints([a, slots[1], b]), ints([b, slots[4], slots[4]])), plain.fork([a, slots[1], b], [b, slots[4], slots[4]]))
        plain.same(c)
        for window, sinks in ((2 * P, 1), (1, P + 1), (P + 6, 0), (1, 0)):
            same_status(c.trim(ints([a, slots[0], a, 77]), window, sinks), plain.trim([a, slots[0], a, 77], window, sinks))
            plain.same(c)
        same_status(c.free(ints([slots[0], slots[0], b, -3])), plain.free([slots[0], slots[0], b, -3]))
        plain.same(c)
        assert int(c.compact()) == plain.compact()
        plain.same(c)
        assert int(c.compact()) == plain.compact()               # nothing left to move
        plain.same(c)
        same_status(c.fork(ints([a, a, a, a]), ints([slots[0], b, slots[4], slots[1]])), plain.fork([a, a, a, a], [slots[0], b, slots[4], slots[1]]))
        plain.same(c)
        same_status(c.free(ints(list(range(7)))), plain.free(list(range(7))))
        assert int(c.compact()) == plain.compact() == 0
        plain.same(c)


def test_many_entries_and_pages(fc):
    """More entries than a workgroup's groups and threads, more pages than one look at the use counts, forks of forty sequences at once, a pool that
    runs out in the middle of a call."""
    import torch
    say("paged bookkeeping, many entries")
    S, N, P = 1500, 9000, 32
    c = fc.PagedCache(N, P, 1, 32, max_seqs=S, max_pages=24)
    c.k.copy_(torch.arange(N, device="cuda").view(1, N, 1, 1, 1) % 251), c.v.copy_(c.k * 2)
    plain, rnd = Plain(c), random.Random(1)
    seqs = rnd.sample(range(S), S)
    rows = [rnd.choice((0, 1, 31, 32, 33, 300)) for _ in seqs]
    same_status(c.grow(ints(seqs), ints(rows)), plain.grow(seqs, rows))
    same_status(c.advance(ints(seqs), ints(rows)), plain.advance(seqs, rows))
    gone = rnd.sample(range(S), 700)
    same_status(c.free(ints(gone)), plain.free(gone))
    src = [s for s in range(S) if s not in set(gone)][:300] * 2
    same_status(c.fork(ints(src), ints(gone[:600])), plain.fork(src, gone[:600]))
    rows = [rnd.choice((0, 1, 64, 400)) for _ in seqs]
    same_status(c.grow(ints(seqs), ints(rows)), plain.grow(seqs, rows))
    gone = rnd.sample(range(S), 900)
    same_status(c.free(ints(gone)), plain.free(gone))
    assert int(c.compact()) == plain.compact()
    assert c.table.tolist() == plain.table and c.ref.tolist() == plain.ref and c.len.tolist() == plain.len
    assert torch.equal(c.k, plain.k) and torch.equal(c.v, plain.v)


def test_serving_loop(fc):
    """The calls as a serving loop makes them: prompts come in, steps grow, write, attend and commit, one sequence is continued twice, a window gives pages
    back, sequences end, the pool is moved together; then a step as one graph, replayed between the program's own work."""
    import torch
    say("paged serving loop")
    P, H, Hkv, Dh, S, W, window, sinks = 32, 4, 2, 128, 6, 4, 60, 3
    c = fc.PagedCache(24, P, Hkv, Dh, n_layers=2, max_seqs=S, max_pages=16)
    c.k.fill_(float("nan")), c.v.fill_(float("nan"))
    plain, rnd, seed = Plain(c), random.Random(3), [10]

    def step(seqs, rows, accepted):
        n = max(rows)
        same_status(c.grow(ints(seqs), ints(rows)), plain.grow(seqs, rows))
        for layer in (0, 1):
            seed[0] += 3
            k, v, q = (queries(rows, h, Dh, "f32", seed[0] + i) for i, h in enumerate((Hkv, Hkv, H)))
            where = dict(layer=layer, seqs=ints(seqs), row_start=starts(rows), max_rows=n)
            c.write(k, v, **where)
            plain.write(Dh, layer, seqs, rows, k, v)
            out, lse = c.attn(q, window=window, sinks=sinks, want_lse=True, **where)
            check(out, lse, plain.attn(Dh, layer, seqs, rows, q, window, sinks), "f32")
        same_status(c.advance(ints(seqs), ints(accepted)), plain.advance(seqs, accepted))
        same_status(c.trim(ints(seqs), window, sinks), plain.trim(seqs, window, sinks))
        plain.same(c)

    step([4, 1], [75, 33], [75, 33])
    for _ in range(3):
        step([1, 4], [W, W], [rnd.randint(1, W), rnd.randint(1, W)])
    same_status(c.fork(ints([4, 4]), ints([0, 5])), plain.fork([4, 4], [0, 5]))
    for i in range(3):
        step([0, 1, 4, 5], [W] * 4, [rnd.randint(1, W) for _ in range(4)])
    same_status(c.free(ints([4, 1])), plain.free([4, 1]))
    assert int(c.compact()) == plain.compact()
    step([5, 0, 2], [W, W, 50], [1, W, 50])

    # one more step as a graph: the same calls, tables and lengths moving on between replays
    seqs, rows, acc = ints([2, 0, 5]), ints([W] * 3), ints([2, 1, W])
    k, v, q = (queries([W] * 3, h, Dh, "f32", 99 + h) for h in (Hkv, Hkv, H))
    book = c.book.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.attn(q, seqs=seqs)
    side.synchronize()
    graph, parts = torch.cuda.CUDAGraph(), {}
    with torch.cuda.graph(graph, stream=side):
        c.grow(seqs, rows)
        c.write(k, v, seqs=seqs)
        parts["out"] = c.attn(q, seqs=seqs, window=window, sinks=sinks)
        c.advance(seqs, acc)
        c.trim(seqs, window, sinks)
    assert torch.equal(c.book, book)
    for _ in range(4):
        k.add_(0.25), q.mul_(1.1)
        plain.grow([2, 0, 5], [W] * 3)
        plain.write(Dh, 0, [2, 0, 5], [W] * 3, k, v)
        want = plain.attn(Dh, 0, [2, 0, 5], [W] * 3, q, window, sinks)[0]
        plain.advance([2, 0, 5], [2, 1, W])
        plain.trim([2, 0, 5], window, sinks)
        graph.replay()
        torch.cuda.synchronize()
        assert rel(parts["out"], want) < 2e-6
        plain.same(c)


@pytest.mark.parametrize("B,lo,hi,rows,H,Hkv,Dh,P,cache,act,window,sinks", [
    (1, 5000, 5000, 1, 8, 1, 128, 64, "bf16", "bf16", 0, 0),             # many parts of one unit
    (1, 3001, 3001, 9, 4, 2, 64, 32, "f32", "f32", 0, 0),
    (70, 0, 900, 1, 4, 4, 128, 32, "bf16", "f32", 0, 0),                 # more sequences than lanes, parts that begin and end inside units
    (130, 0, 400, 3, 2, 1, 32, 32, "bf16", "f32", 100, 2),
    (5, 100, 3000, 7, 16, 2, 96, 128, "bf16", "bf16", 700, 40),
    (3, 10, 2000, 300, 4, 2, 128, 64, "bf16", "f32", 0, 0),              # more than four tiles of a sequence
    (2, 700, 1500, 90, 16, 1, 64, 64, "bf16", "bf16", 333, 7),
    (2, 10, 1000, 130, 4, 4, 256, 64, "f32", "f32", 0, 0),
])
def test_attention_in_parts(fc, B, lo, hi, rows, H, Hkv, Dh, P, cache, act, window, sinks):
    """Units that several workgroups share, joined in memory: the same bits in every call, and a scratch that is as it was afterwards."""
    import torch
    say(f"paged attention in parts B={B} {lo}..{hi} rows={rows} H={H}/{Hkv} Dh={Dh} {cache} {act} window={window}")
    rnd = random.Random(B)
    lens = [rnd.randint(lo, hi) for _ in range(B)]
    n_rows = [rows] * B if B < 3 else [rnd.randint(0, rows) for _ in range(B - 1)] + [rows]
    c, slots = make(fc, lens, n_rows, P, Hkv, Dh, cache)
    q = queries(n_rows, H, Dh, act)
    where = dict(seqs=ints(slots), row_start=starts(n_rows), max_rows=rows, window=window, sinks=sinks, want_lse=True)
    out, lse = c.attn(q, **where)
    check(out, lse, dense(c, slots, n_rows, q, window, sinks), act)
    for _ in range(3):
        again, lse2 = c.attn(q, **where)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


def dense(c, slots, rows, q, window, sinks):
    """Plain.attn with a matrix for each sequence and head."""
    import torch
    Dh, P = q.shape[2], c._desc.page_size
    kc, vc = canonical(c.k, Dh)[0][0], canonical(c.v, Dh)[1][0]
    H, G = q.shape[1], q.shape[1] // kc.shape[1]
    out, lse, x = torch.zeros(sum(rows), H, Dh, dtype=torch.float64, device="cuda"), torch.zeros(sum(rows), H, dtype=torch.float64, device="cuda"), 0
    for s, r in zip(slots, rows):
        n = int(c.len[s])
        key, pos = torch.arange(n + r, device="cuda"), torch.arange(n, n + r, device="cuda")[:, None]
        pages = c.table[s].long()[key // P]
        hidden = (key > pos) | (pages < 0)
        if window:
            hidden |= (key <= pos - window) & (key >= sinks)
        for h in range(H if r else 0):
            k, v = (x_[pages.clamp(min=0), h // G, key % P].double() for x_ in (kc, vc))
            score = (q[x:x + r, h].double() @ k.T / Dh ** 0.5).masked_fill(hidden, -torch.inf)
            lse[x:x + r, h] = torch.logsumexp(score, 1)
            out[x:x + r, h] = torch.softmax(score, 1) @ v
        x += r
    return out.view(sum(rows), -1), lse
