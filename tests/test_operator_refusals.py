"""What the operators for many requests refuse, before any device call (no GPU): argument checks of the C entries, and the host
arithmetic that their kernels share work by."""
import ctypes as C

import pytest
import torch

from paper_2406_13170_b200 import binding as b
from paper_2406_13170_b200 import build as amph_build

P = 0x10000          # an address that is never used: every call below is refused by the host


@pytest.fixture(scope="module")
def L():
    amph_build.build()
    return b.lib()


def _message(L):
    return L.amph_last_error(None).decode()


def _cache(**kw):
    c = dict(k_pages=P, v_pages=P, dtype=1, n_kv_heads=4, head_dim=128, page_size=16, n_pages=10)
    c.update(kw)
    return b.amph_paged_cache(**c)


CACHE_FAULTS = [(dict(k_pages=None), 1), (dict(v_pages=None), 1), (dict(dtype=2), 2), (dict(head_dim=96), 2), (dict(n_kv_heads=0), 2),
                (dict(n_pages=0), 2), (dict(page_size=24), 2), (dict(page_size=0), 2), (dict(page_size=-16), 2), (dict(page_size=1 << 17), 2),
                (dict(k_pages=P + 8), 1)]


def _attend(L, cache=None, q=P, n_heads=8, lens=P, table=P, n_seqs=3, stride=4, scale=0.0, out=2 * P, ws=P, ws_bytes=b.AMPH_PAGED_WS_BYTES):
    cache = _cache() if cache is None else cache
    return L.amph_paged_attention(C.byref(cache) if cache else None, q, n_heads, lens, table, n_seqs, stride, scale, out, None, ws, ws_bytes, 0,
                                  None, None)


@pytest.mark.parametrize("fault,status", CACHE_FAULTS)
def test_attention_and_write_refuse_caches(L, fault, status):
    assert _attend(L, _cache(**fault)) == status
    assert _write(L, _cache(**fault)) == status
    assert _message(L)


def test_pages_that_32_byte_loads_cannot_take(L):
    for fault in (dict(k_pages=P + 16), dict(v_pages=P + 16)):
        assert _attend(L, _cache(**fault)) == 1 and "32-byte" in _message(L)


@pytest.mark.parametrize("fault,status", [
    (dict(q=None), 1), (dict(lens=None), 1), (dict(table=None), 1), (dict(out=None), 1), (dict(out=P), 1), (dict(q=P + 2), 1),
    (dict(n_heads=0), 2), (dict(n_heads=6), 2), (dict(n_heads=2048), 2), (dict(n_seqs=-1), 2), (dict(n_seqs=4097), 2), (dict(stride=0), 2),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(ws=None), 5), (dict(ws=P + 128), 5), (dict(ws_bytes=1000), 5)])
def test_attention_refuses(L, fault, status):
    assert _attend(L, **fault) == status
    assert _message(L)


@pytest.mark.parametrize("dtype,bytes_", [(1, 2), (0, 4)])
@pytest.mark.parametrize("n_seqs", [1, 3, 4096])
def test_attention_refuses_an_output_that_overlaps_its_queries(L, n_seqs, dtype, bytes_):
    """Rows of one sequence are written while another's are still read."""
    size = n_seqs * 8 * 128 * bytes_
    far = 1 << 32
    for by in (16, size // 2, size - 16):
        for out in (far + by, far - by):
            assert _attend(L, _cache(dtype=dtype), q=far, out=out, n_seqs=n_seqs) == 1 and "overlap" in _message(L)
    for out in (far + size, far - size):
        assert _attend(L, _cache(dtype=dtype), q=far, out=out, n_seqs=n_seqs, ws=None) == 5       # (refused for another reason: no launch)


@pytest.mark.parametrize("scale", [2.5e38, -2.5e38, 3.4e38])
def test_attention_refuses_scales_that_overflow_in_the_kernel(L, scale):
    """Scores are taken in units of log 2: the scale times log2(e) has to be a number too (an infinite one makes every score of 0 NaN)."""
    assert _attend(L, scale=scale) == 1 and "scale" in _message(L)


def test_null_cache_and_empty_batches(L):
    assert L.amph_paged_attention(None, P, 8, P, P, 3, 4, 0.0, 2 * P, None, P, b.AMPH_PAGED_WS_BYTES, 0, None, None) == 1
    assert _attend(L, n_seqs=0) == 0                  # nothing to do: no launch
    assert _write(L, rows=0) == 0


def _write(L, cache=None, q=P, qs=1024, k=P, ks=512, v=P, vs=512, src=1, n_heads=8, rows=5, seq=P, pos=P, table=P, n_seqs=3, stride=4,
           theta=10000.0, q_out=P):
    cache = _cache() if cache is None else cache
    return L.amph_paged_write(C.byref(cache), q, qs, k, ks, v, vs, src, n_heads, rows, seq, pos, table, n_seqs, stride, theta, q_out, None, None)


@pytest.mark.parametrize("fault,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(seq=None), 1), (dict(pos=None), 1), (dict(table=None), 1), (dict(q=None), 1),
    (dict(q_out=None), 1), (dict(n_heads=0), 1), (dict(q=None, q_out=None), 1), (dict(q=P + 4), 1), (dict(k=P + 8), 1), (dict(v=P + 8), 1),
    (dict(q_out=P + 8), 1), (dict(ks=516), 1), (dict(qs=1023), 2), (dict(ks=256), 2), (dict(vs=0), 2), (dict(src=3), 2), (dict(rows=-1), 2),
    (dict(n_heads=2000, qs=2000 * 128), 2), (dict(theta=0.0), 1), (dict(theta=-1.0), 1), (dict(theta=float("nan")), 1),
    (dict(theta=float("inf")), 1), (dict(stride=0), 2), (dict(n_seqs=-1), 2)])
def test_write_refuses(L, fault, status):
    assert _write(L, **fault) == status
    assert _message(L)


def _project(L, x=P, cap=16, w=P, n_seg=2, out=256, in_=128, rows=5, dtype=1, tc=1, ad=True, row_adapter=P, y=P, y_dtype=1, ws=P, ws_bytes=1 << 40,
             **kw):
    a = dict(a=P, b=P, scale=None, n_adapters=3, rank=16)
    a.update(kw)
    arr = (C.c_void_p * 8)(*[w] * 8)
    return L.amph_project_adapters(x, cap, arr, n_seg, out, in_, rows, dtype, tc, C.byref(b.amph_adapters(**a)) if ad else None, row_adapter, y,
                                   y_dtype, ws, ws_bytes, None, None)


@pytest.mark.parametrize("fault,status", [
    (dict(x=None), 1), (dict(w=None), 1), (dict(ad=False), 1), (dict(a=None), 1), (dict(b=None), 1), (dict(row_adapter=None), 1), (dict(y=None), 1),
    (dict(x=P + 8), 1), (dict(w=P + 8), 1), (dict(a=P + 8), 1), (dict(b=P + 8), 1), (dict(y=P + 8), 1),
    (dict(n_seg=0), 2), (dict(n_seg=9), 2), (dict(out=0), 2), (dict(in_=4), 2), (dict(in_=132), 2), (dict(rows=0), 2), (dict(rows=513, cap=640), 2),
    (dict(cap=4), 2), (dict(dtype=2), 2), (dict(dtype=0, tc=0), 2), (dict(y_dtype=2), 2), (dict(rank=0), 2), (dict(rank=12), 2), (dict(rank=136), 2),
    (dict(n_adapters=0), 2), (dict(dtype=0, y_dtype=0), 2), (dict(out=200), 2), (dict(in_=136), 2), (dict(cap=15), 2),
    (dict(ws=None), 5), (dict(ws=P + 64), 5), (dict(ws_bytes=1000), 5)])
def test_project_adapters_refuses(L, fault, status):
    assert _project(L, **fault) == status
    assert _message(L)


def test_project_adapters_bytes(L):
    n = C.c_size_t()
    for args in [(0, 128, 1, 16), (9, 128, 1, 16), (1, 0, 1, 16), (1, 128, 0, 16), (1, 128, 513, 16), (1, 128, 1, 4), (1, 128, 1, 20)]:
        assert L.amph_project_adapters_bytes(*args, C.byref(n)) == 2
    assert L.amph_project_adapters_bytes(1, 128, 1, 16, None) == 1
    assert L.amph_project_adapters_bytes(3, 4096, 512, 128, C.byref(n)) == 0
    assert n.value >= 512 * 3 * 4096 * 4 + 512 * 3 * 128 * 4 and n.value % 256 == 0


def test_no_device_means_error(L):
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    assert _attend(L) == 7 and _write(L) == 7 and _project(L) == 7


def test_python_entries_refuse_host_tensors():
    pages = torch.zeros(4, 2, 16, 64)
    with pytest.raises(b.AmphError) as e:
        b.PagedCache(pages, pages.clone())
    assert e.value.status == 7
    with pytest.raises(b.AmphError) as e:
        b.PagedCache(pages.half(), pages.half())
    assert e.value.status == 2
    with pytest.raises(b.AmphError) as e:
        b.Adapters(torch.zeros(2, 1, 8, 64), torch.zeros(2, 1, 64, 16))
    assert e.value.status == 2
    with pytest.raises(b.AmphError) as e:
        b.Adapters(torch.zeros(2, 1, 8, 64), torch.zeros(2, 1, 64, 8))
    assert e.value.status == 7


@pytest.mark.parametrize("head_dim", [0, 1, 32, 96, 256])
def test_a_cache_of_other_head_sizes_cannot_be_made(head_dim):
    """Refused before the device is looked at: paged_write counts q's heads by it."""
    for dtype in (torch.float32, torch.bfloat16):
        pages = torch.zeros(4, 2, 16, head_dim, dtype=dtype)
        with pytest.raises(b.AmphError, match="head_dim") as e:
            b.PagedCache(pages, pages.clone())
        assert e.value.status == 2


@pytest.mark.parametrize("n", [1, 2, 3, 7, 148, 444, 592])
def test_units_spread_over_blocks(n):
    """Block c takes units [total c / n, total (c + 1) / n); block_of() of the attention kernel names the block of a unit."""
    for total in [n, n + 1, 2 * n - 1, 1000, 1001, 12345, 99991]:
        if total < n:
            continue
        owner = {}
        for c in range(n):
            u0, u1 = total * c // n, total * (c + 1) // n
            assert u1 > u0
            for u in range(u0, u1):
                owner[u] = c
        assert len(owner) == total
        for u in range(total):
            assert ((u + 1) * n - 1) // total == owner[u]
