"""The operators for many requests at the ends of what they take."""
import pytest
import torch

from tests.test_gpu_adapters import DEV, _cap, _definition, _ints
from tests.test_gpu_paged import _check_attention, _gen, _near, _normal, _rotated, _table

pytestmark = pytest.mark.gpu
both = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])


@both
@pytest.mark.parametrize("heads,kv,dh,page,lens,width", [
    (2, 1, 64, 8, [(i * 29) % 40 for i in range(4096)], None),          # the most sequences
    (2, 1, 64, 8, [0] * 4095 + [33], None),                             # one among the most that has keys
    (2, 2, 128, 1, [0] * 4096, None),                                   # none
    (1024, 1024, 64, 16, [17, 0, 1], None),                             # the most heads, each with keys of its own
    (1024, 1, 128, 16, [70], None),                                     # sharing one: 128 items
    (1024, 8, 64, 4, [3, 300], 5000),
    (8, 2, 64, 65536, [1, 65536, 65537, 70000], None),                  # the largest pages
    (1, 1, 64, 1, [1], 1 << 20),                                        # the widest row of a table here
    (1, 1, 128, 65536, [5], 1 << 15),                                   # room for 2^31 positions
])
def test_attention_at_its_limits(dtype, heads, kv, dh, page, lens, width):
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(heads + len(lens))
    table, n_pages = _table(lens, page, g, width=width, spare=1)
    kp, vp = _normal(g, n_pages, kv, page, dh, dtype=dtype), _normal(g, n_pages, kv, page, dh, dtype=dtype)
    q = _normal(g, len(lens), heads, dh, dtype=dtype)
    lse = torch.empty(len(lens), heads, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse, status=status)
    assert int(status) == 0
    _check_attention(out, lse, q, kp, vp, table, lens)


@both
@pytest.mark.parametrize("heads,kv,dh,rows", [(1024, 1024, 64, 3), (1024, 1, 128, 20), (1, 1, 64, 70000), (4, 2, 128, 33000), (0, 1024, 64, 5)])
def test_write_at_its_limits(dtype, heads, kv, dh, rows):
    from paper_2406_13170_b200 import PagedCache, paged_write
    g = _gen(rows)
    table, n_pages = _table([rows], 16, g)
    kp, vp = (torch.zeros(n_pages, kv, 16, dh, dtype=dtype, device=DEV) for _ in range(2))
    q = _normal(g, rows, heads * dh, dtype=torch.bfloat16) if heads else None
    k, v = _normal(g, rows, kv * dh, dtype=torch.bfloat16), _normal(g, rows, kv * dh, dtype=torch.bfloat16)
    pos = torch.randperm(rows, generator=g, device=DEV).to(torch.int32)
    out = paged_write(PagedCache(kp, vp), q, k, v, torch.zeros_like(pos), pos, table)
    at = pos.long()
    pages = table[0, at // 16].long()
    want, size = _rotated(k, at, kv, dh, 10000.0)
    assert _near(kp[pages, :, at % 16], want, size)
    assert torch.equal(vp[pages, :, at % 16], v.view(rows, kv, dh).to(dtype))
    if heads:
        want, size = _rotated(q, at, heads, dh, 10000.0)
        assert _near(out, want, size)


@pytest.mark.parametrize("rows,n_seg,out,in_,rank,n,dtype", [
    (512, 8, 512, 256, 128, 3, torch.bfloat16),            # the most rows, matrices and rank
    (512, 8, 512, 256, 128, 700, torch.bfloat16),          # more adapters than rows
    (512, 1, 256, 64, 128, 512, torch.bfloat16),           # an adapter for each row
    (1, 8, 2048, 2048, 128, 1, torch.bfloat16),
    (1, 1, 128, 64, 8, 100000, torch.bfloat16),            # a large pool
    (512, 8, 40, 128, 128, 60, torch.float32),
    (1, 1, 1, 8, 8, 1, torch.bfloat16),                    # the smallest
    (1, 1, 1, 8, 8, 1, torch.float32),
    (512, 1, 32000, 256, 16, 9, torch.bfloat16),           # a vocabulary
    (129, 3, 1152, 704, 40, 20, torch.bfloat16),           # odd numbers of tiles and of K blocks
])
def test_adapters_at_their_limits(rows, n_seg, out, in_, rank, n, dtype):
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(rows + rank)
    x, ws = _ints(g, -1, 1, _cap(rows), in_, dtype=dtype), [_ints(g, -2, 2, out, in_, dtype=dtype) for _ in range(n_seg)]
    a, b = _ints(g, -1, 1, n, n_seg, rank, in_, dtype=dtype), _ints(g, -2, 2, n, n_seg, out, rank, dtype=dtype)
    tc = dtype is torch.bfloat16 and out % 128 == 0 and in_ % 64 == 0
    for at in (torch.randint(-1, n, (rows,), generator=g, device=DEV), torch.arange(rows, device=DEV) % n, torch.full((rows,), n - 1, device=DEV)):
        at = at.to(torch.int32)
        y = project_adapters(x, ws, rows, tc, Adapters(a, b), at, y_dtype=torch.float32)
        want = _definition(x, ws, a, b, None, at.tolist())
        assert float(want.abs().max()) < 2 ** 23 and torch.equal(y.double(), want)
