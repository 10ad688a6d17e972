"""Host-only checks of the paged cache's entry points: sizes, and the refusals that come before any launch."""
import ctypes

import pytest

from paper_2311_08263_amd import binding
from paper_2311_08263_amd.binding import PagedDesc, PagedRows

EINVAL = -1


def desc(**kw):
    d = dict(n_layers=2, n_pages=10, page_size=64, n_kv_heads=4, head_dim=128, dtype=1, max_seqs=3, max_pages=5, k_pool=1 << 20, v_pool=1 << 21, table=4096, len=8192, ref=12288)
    d.update(kw)
    return PagedDesc(*(d[n] for n, _ in PagedDesc._fields_))


def refused(rc, text):
    assert rc == EINVAL and text in binding.lib().fastcot_last_error(None), binding.lib().fastcot_last_error(None)


def test_sizes():
    L = binding.lib()
    assert L.fastcot_paged_pool_bytes(ctypes.byref(desc())) == 2 * 10 * 64 * 4 * 128 * 2
    assert L.fastcot_paged_pool_bytes(ctypes.byref(desc(dtype=0, head_dim=96))) == 2 * 10 * 64 * 4 * 96 * 4
    assert L.fastcot_paged_pool_bytes(ctypes.byref(desc(n_pages=1 << 20, page_size=4096, max_pages=1, n_layers=80))) == 80 * (1 << 20) * 4096 * 4 * 128 * 2
    assert L.fastcot_paged_scratch_bytes(ctypes.byref(desc())) > 0


def test_more_blocks_than_31_bits_count():
    """Rows times positions of the table, which the kernel deals out by number."""
    r = PagedRows(3, 1 << 20, 3 << 20, None, None)
    assert attn(d=desc(max_pages=1 << 24), r=r) == -3 and b"2^31" in binding.lib().fastcot_last_error(None)
    assert attn(r=PagedRows(1, 1 << 26, 1 << 26, None, None)) == -3


BAD = [dict(n_layers=4096, n_kv_heads=4096, page_size=4096), dict(n_layers=0), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(page_size=16), dict(page_size=48), dict(page_size=8192), dict(n_kv_heads=0),
       dict(head_dim=100), dict(head_dim=160), dict(dtype=2), dict(max_seqs=0), dict(max_seqs=4097), dict(max_pages=0), dict(max_pages=1 << 25),
       # table entries past 31 bits, bytes of a pool past 64
       dict(max_seqs=128, max_pages=1 << 24), dict(n_layers=512, n_pages=1 << 24, n_kv_heads=1024, page_size=4096, max_pages=1),
       dict(n_layers=128, n_pages=1 << 24, n_kv_heads=4096, page_size=1024, head_dim=256, dtype=0, max_pages=1)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_bad_descriptions(bad):
    L = binding.lib()
    d = ctypes.byref(desc(**bad))
    assert L.fastcot_paged_pool_bytes(d) == 0 and L.fastcot_paged_scratch_bytes(d) == 0
    refused(L.fastcot_paged_reset(d, None), b"fastcot_paged_reset: bad cache description")
    refused(L.fastcot_paged_grow(d, 1, 4096, 4096, None, 4096, None), b"bad cache description")


def test_missing_and_misaligned_memory():
    L = binding.lib()
    for name in ("k_pool", "v_pool", "table", "len", "ref"):
        refused(L.fastcot_paged_compact(ctypes.byref(desc(**{name: None})), None, 4096, None), b"NULL")
    refused(L.fastcot_paged_compact(ctypes.byref(desc(k_pool=4104)), None, 4096, None), b"16 bytes")
    refused(L.fastcot_paged_compact(ctypes.byref(desc(ref=4097)), None, 4096, None), b"misaligned")
    refused(L.fastcot_paged_compact(ctypes.byref(desc()), None, None, None), b"scratch")
    refused(L.fastcot_paged_compact(ctypes.byref(desc()), None, 4160, None), b"scratch")
    refused(L.fastcot_paged_reset(None, None), b"bad cache description")


def test_entries():
    L, d = binding.lib(), ctypes.byref(desc())
    for count in (-1, 4):
        refused(L.fastcot_paged_grow(d, count, 4096, 4096, None, 4096, None), b"count")
        refused(L.fastcot_paged_advance(d, count, 4096, 4096, None, None), b"count")
        refused(L.fastcot_paged_fork(d, count, 4096, 4096, None, 4096, None), b"count")
        refused(L.fastcot_paged_free(d, count, 4096, None, None), b"count")
        refused(L.fastcot_paged_trim(d, count, 4096, 5, 0, None, None), b"count")
    refused(L.fastcot_paged_grow(d, 1, None, 4096, None, 4096, None), b"NULL")
    refused(L.fastcot_paged_grow(d, 1, 4097, 4096, None, 4096, None), b"misaligned")
    refused(L.fastcot_paged_advance(d, 1, 4096, None, None, None), b"NULL")
    refused(L.fastcot_paged_grow(d, 1, 4096, 4096, None, None, None), b"scratch")
    refused(L.fastcot_paged_fork(d, 1, 4096, 4096, None, None, None), b"scratch")
    refused(L.fastcot_paged_trim(d, 1, 4096, 0, 0, None, None), b"window")
    refused(L.fastcot_paged_trim(d, 1, 4096, 1, -1, None, None), b"sinks")
    # nothing to do: no launch
    assert L.fastcot_paged_grow(d, 0, None, None, None, 4096, None) == 0
    assert L.fastcot_paged_advance(d, 0, None, None, None, None) == 0
    assert L.fastcot_paged_fork(d, 0, None, None, None, 4096, None) == 0
    assert L.fastcot_paged_trim(d, 0, None, 1, 0, None, None) == 0
    assert L.fastcot_paged_free(d, 0, None, None, None) == 0


def attn(d=None, r=None, layer=0, q=4096, qr=4096, qh=128, H=32, act=0, window=0, sinks=0, out=4096, orow=4096, scratch=4096):
    r = PagedRows(3, 2, 6, None, None) if r is None else r
    return binding.lib().fastcot_paged_attn(ctypes.byref(d or desc()), layer, ctypes.byref(r), q, qr, qh, H, act, window, sinks, out, orow, None, scratch, None)


def write(d=None, r=None, layer=0, k=4096, v=4096, row=512, act=1):
    r = PagedRows(3, 2, 6, None, None) if r is None else r
    return binding.lib().fastcot_paged_write(ctypes.byref(d or desc()), layer, ctypes.byref(r), k, v, row, act, None)


@pytest.mark.parametrize("call", [attn, write])
def test_rows(call):
    refused(call(r=PagedRows(-1, 1, 1, None, None)), b"bad rows")
    refused(call(r=PagedRows(1, -1, 1, None, None)), b"bad rows")
    refused(call(r=PagedRows(1, 1, -1, None, None)), b"bad rows")
    refused(call(r=PagedRows(3, 2, 7, None, None)), b"n_rows")
    refused(call(r=PagedRows(4, 1, 4, None, None)), b"more sequences")
    refused(call(r=PagedRows(70000, 1, 70000, 4096, None)), b"65535")
    refused(call(r=PagedRows(3, 2, 6, 4098, None)), b"misaligned")
    refused(call(r=PagedRows(3, 2, 6, 4096, 4097)), b"misaligned")
    refused(call(layer=2), b"layer")
    refused(call(layer=-1), b"layer")
    refused(call(act=3), b"type")
    refused(call(d=desc(dtype=0), act=1), b"fp32 cache")
    for r in (PagedRows(0, 0, 0, None, None), PagedRows(3, 0, 0, None, None), PagedRows(3, 5, 0, 4096, 4096)):
        assert call(r=r) == 0                  # no rows: no launch


def test_attention_arguments():
    refused(attn(H=0), b"heads")
    refused(attn(H=30), b"heads")
    refused(attn(H=4 * 65), b"heads")
    refused(attn(window=-1), b"window")
    refused(attn(sinks=-1), b"sinks")
    refused(attn(q=None), b"queries")
    refused(attn(out=None), b"queries")
    refused(attn(q=4104), b"16 bytes")
    refused(attn(out=4100), b"16 bytes")
    refused(attn(qr=4097), b"strides")
    refused(attn(qh=-128), b"strides")
    refused(attn(orow=4088), b"output")
    refused(attn(orow=4100), b"output")
    refused(attn(scratch=None), b"scratch")


def test_write_arguments():
    refused(write(k=None), b"K and V")
    refused(write(v=4104), b"16 bytes")
    refused(write(row=504), b"stride")
    refused(write(row=516), b"stride")
    assert write(r=PagedRows(1, (1 << 30) + 1, (1 << 30) + 1, None, None)) == -3 and b"too many rows" in binding.lib().fastcot_last_error(None)
