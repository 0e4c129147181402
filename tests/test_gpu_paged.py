"""Paged caches: writing rows into their pages, and the attention of one new token, against plain definitions in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}        # half a step of the output's type, relative (fp32's is part of the sums)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=torch.float32, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _table(lens, page, g, width=None, spare=2):
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=g, device=DEV).tolist()
    width = width or max(1, max(need))
    rows, at = [], 0
    for n in need:
        rows.append(order[at: at + n] + [-7] * (width - n))
        at += n
    return torch.tensor(rows, dtype=torch.int32, device=DEV), n_pages


def _gathered(pages, table_row, n):
    """[n, kv, dh] of a sequence in 64 bits."""
    page = pages.shape[2]
    at = torch.arange(n, device=DEV)
    return pages[table_row.long()[at // page], :, at % page].double()


def _reference(q, k_pages, v_pages, table, lens, scale=None):
    """(out, lse, weighted mean of |v|, largest sum of |q k| scale) per sequence and head, in 64 bits."""
    n, heads, dh = q.shape
    kv = k_pages.shape[1]
    scale = dh ** -0.5 if scale is None else scale
    o = torch.zeros(n, heads, dh, dtype=torch.float64, device=DEV)
    a, lse = torch.zeros_like(o), torch.full((n, heads), -math.inf, dtype=torch.float64, device=DEV)
    mass = torch.zeros(n, heads, dtype=torch.float64, device=DEV)
    for s, m in enumerate(lens):
        if m <= 0:
            continue
        k, v = _gathered(k_pages, table[s], m), _gathered(v_pages, table[s], m)
        qs = q[s].double().reshape(kv, heads // kv, dh)
        z = torch.einsum("hgd,nhd->hgn", qs, k) * scale
        w = torch.softmax(z, -1)
        o[s] = torch.einsum("hgn,nhd->hgd", w, v).reshape(heads, dh)
        a[s] = torch.einsum("hgn,nhd->hgd", w, v.abs()).reshape(heads, dh)
        lse[s] = torch.logsumexp(z, -1).reshape(heads)
        mass[s] = (torch.einsum("hgd,nhd->hgn", qs.abs(), k.abs()).amax(-1) * abs(scale)).reshape(heads)
    return o, lse, a, mass


def _check_attention(out, lse, q, k_pages, v_pages, table, lens, scale=None):
    """Scores: sums of head_dim products (at most head_dim roundings of 2 u on the tensor cores' truncating sums) on sum |q k|, two
    more for the scale; weights: exp2 to 2 ulp, rescaled once per 16 keys of a warp, 16 bits of them enter the second product on tensor cores (2^-16);
    weighted values: a sum over the keys.  Every weight's relative error enters numerator and denominator."""
    o, l, a, mass = _reference(q, k_pages, v_pages, table, lens, scale)
    dh = q.shape[2]
    n = torch.tensor([max(m, 0) for m in lens], dtype=torch.float64, device=DEV)[:, None]
    score = (2 * dh + 4) * U * mass
    eps = score + (n / 64 + 8) * 4 * U + 2.0 ** -16 + 2 * U * n
    tol = 2 * eps[..., None] * a + (HALF[out.dtype] + U) * o.abs()
    bad = ~((out.double() - o).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {float(((out.double() - o).abs() / tol.clamp(min=1e-300)).max())} of the tolerance"
    if lse is not None:
        empty = torch.isinf(l)
        assert torch.equal(torch.isinf(lse), empty)
        assert bool((((lse.double() - l).abs() <= 2 * eps + 4 * U * l.abs()) | empty).all())


# heads, kv heads, head_dim, page, lengths
ATTEND = [
    (4, 4, 64, 16, [1]),
    (4, 4, 64, 16, [0, 1, 15, 16, 17, 31, 33, 63, 64, 65]),
    (32, 32, 128, 16, [640]),
    (32, 8, 128, 16, [0, 5, 0, 300, 129, 1, 0]),
    (40, 40, 128, 64, [90, 700, 2048]),
    (8, 8, 128, 1, [1, 2, 77, 130]),               # a page per token
    (8, 2, 64, 2, [3, 64, 190]),
    (5, 1, 64, 8, [7, 8, 9, 500]),                 # five heads share one
    (16, 2, 128, 8, [61, 4097]),
    (12, 1, 128, 32, [1000, 31]),                  # twelve heads share one: more than a block of eight
    (71, 1, 64, 16, [333]),
    (52, 52, 128, 256, [100, 256, 257]),
    (8, 1, 128, 1024, [5000]),
    (64, 8, 128, 16, [20011]),                     # one sequence over every block
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,dh,page,lens", ATTEND)
def test_attention(dtype, heads, kv, dh, page, lens):
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(heads * 131 + len(lens))
    table, n_pages = _table(lens, page, g)
    kp, vp = _normal(g, n_pages, kv, page, dh, dtype=dtype), _normal(g, n_pages, kv, page, dh, dtype=dtype)
    q = _normal(g, len(lens), heads, dh, dtype=dtype, std=2.0)
    lse = torch.full((len(lens), heads), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse, status=status)
    assert out.dtype is dtype and int(status) == 0
    _check_attention(out, lse, q, kp, vp, table, lens)
    again = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,dh,page,lens", ATTEND)
def test_short_sequences_in_wide_tables(dtype, heads, kv, dh, page, lens):
    """The table's width chooses the kernel: these have room for 150,000 tokens."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(heads * 17 + len(lens))
    table, n_pages = _table(lens, page, g, width=-(-150000 // page))
    kp, vp = _normal(g, n_pages, kv, page, dh, dtype=dtype), _normal(g, n_pages, kv, page, dh, dtype=dtype)
    q = _normal(g, len(lens), heads, dh, dtype=dtype, std=2.0)
    lse = torch.full((len(lens), heads), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse, status=status)
    assert int(status) == 0
    _check_attention(out, lse, q, kp, vp, table, lens)
    # absent pages and lengths that do not exist, in this kernel too
    bad = table.clone()
    bad[:, 0] = n_pages
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out2 = paged_attention(PagedCache(kp, vp), q, bad, n, status=status)
    assert int(status) == (1 if max(lens) > 0 else 0) and torch.isfinite(out2.float()).all()
    n[-1] = -5
    status.zero_()
    out2 = paged_attention(PagedCache(kp, vp), q, table, n, status=status)
    assert int(status) == 1 and not out2[-1].any() and torch.equal(out2[:-1], paged_attention(PagedCache(kp, vp), q, table, n)[:-1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,dh,page,lens", [       # items cut into hundreds of parts, and into a few with whole ones around them
    (8, 1, 128, 32, [40001]), (1, 1, 64, 64, [60000]), (5, 1, 128, 16, [1, 30000, 64]), (6, 2, 64, 256, [33333, 0, 2]), (11, 1, 128, 64, [25000]),
    (2, 2, 128, 16, [1500, 64, 9000, 1, 65, 128, 7000, 3] * 3),
])
def test_attention_over_many_parts(dtype, heads, kv, dh, page, lens):
    test_attention(dtype, heads, kv, dh, page, lens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_attention_of_many_sequences(dtype):
    """More sequences than threads in a block, most of them short, some empty; a table wider than any needs; a scale of one's own."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(5)
    lens = [(i * 37) % 150 if i % 5 else 0 for i in range(1111)]
    table, n_pages = _table(lens, 16, g, width=23)
    kp, vp = _normal(g, n_pages, 2, 16, 64, dtype=dtype), _normal(g, n_pages, 2, 16, 64, dtype=dtype)
    q = _normal(g, len(lens), 4, 64, dtype=dtype)
    lse = torch.empty(len(lens), 4, device=DEV)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), scale=0.3, lse=lse)
    _check_attention(out, lse, q, kp, vp, table, lens, scale=0.3)


@pytest.mark.parametrize("scale", [1e-50, -1e-50, 1e-300, 1e-40])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_scales_too_small_to_matter(dtype, scale):
    """Every key has the same weight; 0 in fp32, which stands for 1 / sqrt(head_dim), is not what such a scale becomes."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(19)
    lens = [1, 100, 0, 700]
    table, n_pages = _table(lens, 16, g)
    kp, vp = _normal(g, n_pages, 2, 16, 128, dtype=dtype), _normal(g, n_pages, 2, 16, 128, dtype=dtype)
    q = _normal(g, len(lens), 4, 128, dtype=dtype)
    lse = torch.empty(len(lens), 4, device=DEV)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), scale=scale, lse=lse)
    _check_attention(out, lse, q, kp, vp, table, lens, scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("page", [1, 8, 16, 64])
def test_slots_behind_a_sequence_are_not_looked_at(dtype, page):
    """What lies behind a sequence's last token, in its last page and in pages of others, may be anything: NaN and infinities."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(11)
    lens = [1, 13, 50, 0, 64, 201]
    table, n_pages = _table(lens, page, g)
    kp, vp = (torch.full((n_pages, 2, page, 128), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    vp[1::2] = math.inf
    for s, n in enumerate(lens):
        for t in range(n):
            pg = int(table[s, t // page])
            kp[pg, :, t % page] = _normal(g, 2, 128, dtype=dtype)
            vp[pg, :, t % page] = _normal(g, 2, 128, dtype=dtype)
    q = _normal(g, len(lens), 8, 128, dtype=dtype)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
    _check_attention(out, None, q, kp, vp, table, lens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_scores_of_every_size(dtype):
    """Scores that grow along the sequence (the running maximum moves at every step), that fall, and that differ by more than exp can hold."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(12)
    lens = [300, 300, 300]
    table, n_pages = _table(lens, 16, g)
    kp, vp = torch.zeros(n_pages, 1, 16, 64, dtype=dtype, device=DEV), _normal(g, n_pages, 1, 16, 64, dtype=dtype)
    ramp = torch.arange(300, device=DEV, dtype=torch.float32)
    for s, v in enumerate([ramp / 4, -ramp / 4, torch.where(ramp == 177, 2000.0, -1000.0)]):
        for t in range(300):
            kp[int(table[s, t // 16]), 0, t % 16, :4] = float(v[t])
    q = torch.ones(3, 2, 64, dtype=dtype, device=DEV)
    lse = torch.empty(3, 2, device=DEV)
    out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse)
    _check_attention(out, lse, q, kp, vp, table, lens)


def test_infinite_and_nan_scores():
    """A key of -inf gets no weight; NaN among a sequence's own keys makes its rows NaN, and no other's."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(13)
    lens = [40, 100, 70]
    for dtype in (torch.bfloat16, torch.float32):
        table, n_pages = _table(lens, 16, g)
        kp, vp = _normal(g, n_pages, 1, 16, 64, dtype=dtype), _normal(g, n_pages, 1, 16, 64, dtype=dtype)
        q = torch.ones(3, 1, 64, dtype=dtype, device=DEV)
        kp[int(table[0, 1]), 0, 3] = -math.inf
        kp[int(table[1, 5]), 0, 9] = math.nan
        out = paged_attention(PagedCache(kp, vp), q, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
        assert torch.isnan(out[1]).all() and torch.isfinite(out[0]).all() and torch.isfinite(out[2]).all()
        k0 = _gathered(kp, table[0], 40)[:, 0] .sum(-1) / 8
        ref = torch.softmax(k0, 0) @ _gathered(vp, table[0], 40)[:, 0]
        assert float((out[0, 0].double() - ref).abs().max()) <= 2.0 ** -7 * float(ref.abs().max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("wide", [False, True], ids=["narrow", "wide"])
def test_infinite_values(dtype, wide):
    """An infinity among a sequence's own values makes its column infinite or NaN in the heads that read it, and changes nothing else."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(16)
    lens = [40, 100, 700]
    table, n_pages = _table(lens, 16, g, width=9000 if wide else None)
    kp, vp = _normal(g, n_pages, 2, 16, 64, dtype=dtype), _normal(g, n_pages, 2, 16, 64, dtype=dtype)
    q, n = _normal(g, 3, 8, 64, dtype=dtype), torch.tensor(lens, dtype=torch.int32, device=DEV)
    good = paged_attention(PagedCache(kp, vp), q, table, n)
    vp[int(table[1, 5]), 1, 9, 33] = math.inf
    vp[int(table[2, 40]), 0, 2, 7] = -math.inf
    out = paged_attention(PagedCache(kp, vp), q, table, n)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[1, 4:, 33] = hit[2, :4, 7] = True
    assert not torch.isfinite(out[hit]).any() and torch.equal(out[~hit], good[~hit])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("page", [4, 16])
def test_pages_and_lengths_that_do_not_exist(dtype, page):
    """They are reported, count as absent, and the other sequences' rows are what they are without them."""
    from paper_2406_13170_b200 import PagedCache, paged_attention
    g = _gen(14)
    lens = [100, 90, 80, 70]
    table, n_pages = _table(lens, page, g)
    kp, vp = _normal(g, n_pages, 2, page, 64, dtype=dtype), _normal(g, n_pages, 2, page, 64, dtype=dtype)
    q = _normal(g, 4, 4, 64, dtype=dtype)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    good = paged_attention(PagedCache(kp, vp), q, table, ln, status=status)
    assert int(status) == 0
    for entry in (-1, n_pages, 2 ** 31 - 1, -2 ** 31):
        bad = table.clone()
        bad[1, 2] = entry
        status.zero_()
        out = paged_attention(PagedCache(kp, vp), q, bad, ln, status=status)
        assert int(status) == 1
        for s in (0, 2, 3):
            assert torch.equal(out[s], good[s])
        at = torch.tensor([t for t in range(90) if t // page != 2], device=DEV)
        k, v = (p[table[1].long()[at // page], :, at % page].double() for p in (kp, vp))
        w = torch.softmax(torch.einsum("hgd,nhd->hgn", q[1].double().reshape(2, 2, 64), k) / 8, -1)
        ref = torch.einsum("hgn,nhd->hgd", w, v).reshape(4, 64)
        assert float((out[1].double() - ref).abs().max()) <= 2.0 ** -7 * float(ref.abs().max())
    for n in (-5, table.shape[1] * page + 1, 2 ** 31 - 1):
        wrong = ln.clone()
        wrong[0] = n                                  # sequence 0 is the longest: its table row is full
        status.zero_()
        out = paged_attention(PagedCache(kp, vp), q, table, wrong, status=status)
        assert int(status) == 1
        if n < 0:
            assert not out[0].any()
        else:
            assert torch.isfinite(out[0]).all()
    paged_attention(PagedCache(kp, vp), q, table, wrong)      # without a status word


def test_offsets_beyond_32_bits():
    """Pages whose elements lie more than 2^32 elements behind the first."""
    from paper_2406_13170_b200 import PagedCache, paged_attention, paged_write
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("not enough device memory")
    g = _gen(15)
    n_pages, kv, page, dh = 33000, 8, 128, 128
    kp, vp = (torch.empty(n_pages, kv, page, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert (n_pages - 1) * kv * page * dh > 2 ** 32
    table = torch.tensor([[n_pages - 1, 3], [n_pages - 2, 0]], dtype=torch.int32, device=DEV)
    lens = [200, 129]
    seq = torch.tensor([0] * 200 + [1] * 129, dtype=torch.int32, device=DEV)
    pos = torch.tensor(list(range(200)) + list(range(129)), dtype=torch.int32, device=DEV)
    k, v = _normal(g, 329, kv * dh), _normal(g, 329, kv * dh)
    c = PagedCache(kp, vp)
    assert paged_write(c, None, k, v, seq, pos, table) is None
    assert torch.equal(_gathered(vp, table[0], 200).reshape(200, -1), v[:200].bfloat16().double())
    assert torch.equal(_gathered(vp, table[1], 129).reshape(129, -1), v[200:].bfloat16().double())
    q = _normal(g, 2, 16, dh, dtype=torch.bfloat16)
    out = paged_attention(c, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
    _check_attention(out, None, q, kp, vp, table, lens)


# ---------------------------------------------------------------------------------------------------------------------
# write
# ---------------------------------------------------------------------------------------------------------------------
def _rotated(x, pos, heads, dh, theta):
    """(rotated, |lo| + |hi| of every pair) in 64 bits, as a product of complex numbers."""
    x = x.double().reshape(len(pos), heads, 2, dh // 2)
    freq = torch.tensor([theta ** (-2.0 * i / dh) for i in range(dh // 2)], dtype=torch.float64, device=DEV)
    ang = pos.double()[:, None] * freq
    z = torch.complex(x[:, :, 0].contiguous(), x[:, :, 1].contiguous()) * torch.polar(torch.ones_like(ang), ang)[:, None]
    size = x.abs().sum(2, keepdim=True).expand(-1, -1, 2, -1)
    return torch.cat([z.real, z.imag], -1), size.reshape(len(pos), heads, dh)


def _near(got, want, size):
    """Two products and a sum in fp32 (3 u of |lo| + |hi|), cosine and sine to 2 ulp of an angle that is rounded once (3 u), and the output's type."""
    tol = 6 * U * size + (HALF[got.dtype] + U) * want.abs()
    return bool(((got.double() - want).abs() <= tol).all())


WRITE = [  # heads, kv heads, head_dim, page, (first position, rows) of each sequence
    (4, 4, 64, 16, [(0, 1)]),
    (32, 32, 128, 16, [(511, 1), (0, 1), (15, 1), (16, 1)]),
    (32, 8, 128, 64, [(0, 70), (63, 2), (100000, 1)]),
    (5, 1, 64, 1, [(3, 9), (0, 1)]),
    (40, 40, 128, 256, [(250, 13)]),
    (0, 2, 128, 8, [(5, 30)]),                     # keys and values only
]


@pytest.mark.parametrize("theta", [10000.0, 500000.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("source", [torch.bfloat16, torch.float32], ids=["from_bf16", "from_fp32"])
@pytest.mark.parametrize("heads,kv,dh,page,seqs", WRITE)
def test_write(heads, kv, dh, page, seqs, source, dtype, theta):
    from paper_2406_13170_b200 import PagedCache, paged_write
    g = _gen(heads + 7 * page)
    ends = [p + n for p, n in seqs]
    table, n_pages = _table(ends, page, g)
    kp, vp = _normal(g, n_pages, kv, page, dh, dtype=dtype), _normal(g, n_pages, kv, page, dh, dtype=dtype)
    k_before, v_before = kp.clone(), vp.clone()
    order = [(s, p + i) for s, (p, n) in enumerate(seqs) for i in range(n)]
    order = [order[i] for i in torch.randperm(len(order), generator=torch.Generator().manual_seed(3)).tolist()]
    order = order[:1] + [(-1, 5)] + order[1:] + [(-1, 0), (-3, -9)]           # rows of no sequence between and behind
    seq = torch.tensor([s for s, _ in order], dtype=torch.int32, device=DEV)
    pos = torch.tensor([p for _, p in order], dtype=torch.int32, device=DEV)
    rows = len(order)
    qkv = _normal(g, rows, (heads + 2 * kv) * dh + 64, dtype=source)         # rows of a wider matrix
    q, k, v = qkv[:, : heads * dh], qkv[:, heads * dh: (heads + kv) * dh], qkv[:, (heads + kv) * dh: (heads + 2 * kv) * dh]
    q_out = torch.full((rows, heads, dh), 5.0, dtype=dtype, device=DEV) if heads else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = paged_write(PagedCache(kp, vp), q if heads else None, k, v, seq, pos, table, theta=theta, q_out=q_out, status=status)
    assert r is q_out and int(status) == 0
    real = (seq >= 0).nonzero()[:, 0]
    at, where = pos[real].long(), seq[real].long()
    pages = table[where, at // page].long()
    want, size = _rotated(k[real], at, kv, dh, theta)
    assert _near(kp[pages, :, at % page], want, size)
    assert torch.equal(vp[pages, :, at % page], v[real].reshape(len(real), kv, dh).to(dtype))
    if heads:
        want, size = _rotated(q[real], at, heads, dh, theta)
        assert _near(q_out[real], want, size)
        assert bool((q_out[seq < 0] == 5.0).all())
    for now, before in ((kp, k_before), (vp, v_before)):                      # nothing else was touched
        now = now.clone()
        now[pages, :, at % page] = before[pages, :, at % page]
        assert torch.equal(now, before)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("source", [torch.bfloat16, torch.float32], ids=["from_bf16", "from_fp32"])
@pytest.mark.parametrize("heads,kv,dh,page,seqs", [
    (32, 8, 128, 16, [(0, 333), (70001, 90)]), (5, 1, 64, 32, [(7, 5500)]), (33, 3, 128, 64, [(0, 517)]), (0, 2, 64, 1, [(0, 9500)]),
])
def test_write_of_many_rows(heads, kv, dh, page, seqs, source, dtype):
    test_write(heads, kv, dh, page, seqs, source, dtype, 10000.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,dh,rows", [(32, 8, 128, 1), (5, 1, 64, 7), (40, 40, 128, 64), (32, 8, 128, 900)])
def test_queries_rotated_in_place(heads, kv, dh, rows, dtype):
    from paper_2406_13170_b200 import PagedCache, paged_write
    g = _gen(rows)
    table, n_pages = _table([rows + 40], 16, g)
    kp, vp = (torch.zeros(n_pages, kv, 16, dh, dtype=dtype, device=DEV) for _ in range(2))
    q, k, v = _normal(g, rows, heads, dh, dtype=dtype), _normal(g, rows, kv, dh, dtype=dtype), _normal(g, rows, kv, dh, dtype=dtype)
    seq = torch.where(torch.arange(rows, device=DEV) % 5 == 3, -1, 0).to(torch.int32)
    pos = torch.arange(40, 40 + rows, dtype=torch.int32, device=DEV)
    before = q.clone()
    want = paged_write(PagedCache(kp, vp), q, k, v, seq, pos, table, q_out=before.clone())
    keys = kp.clone()
    kp.zero_()
    assert paged_write(PagedCache(kp, vp), q, k, v, seq, pos, table, q_out=q) is q
    assert torch.equal(q, want) and torch.equal(kp, keys) and torch.equal(q[seq < 0], before[seq < 0])


def test_angles_of_far_positions():
    """Position 2^31 - 2^16: the angle's phase is exact, cosine and sine are those of 64-bit arithmetic on an exact product."""
    from paper_2406_13170_b200 import PagedCache, paged_write
    page, dh = 65536, 64
    kp, vp = (torch.zeros(1, 1, page, dh, device=DEV) for _ in range(2))
    wide = (2 ** 31 - 65536) // page
    table = torch.zeros(1, wide, dtype=torch.int32, device=DEV)
    g = _gen(3)
    pos = torch.tensor([2 ** 31 - 65536 - 1, 1 << 30, 1234567890, 3, 1], dtype=torch.int32, device=DEV)
    k = _normal(g, 5, dh)
    q = _normal(g, 5, dh)
    out = paged_write(PagedCache(kp, vp), q, k, k, torch.zeros(5, dtype=torch.int32, device=DEV), pos, table)
    want, size = _rotated(q, pos, 1, dh, 10000.0)
    # a product of 2^31 in 64 bits is off by 2^-22 of a radian at most: part of the reference's own error
    assert bool(((out.double() - want).abs() <= 6 * U * size + U * want.abs() + 2.0 ** -22 * size).all())


def test_rows_that_do_not_fit_are_reported_and_skipped():
    from paper_2406_13170_b200 import PagedCache, paged_write
    g = _gen(4)
    kp, vp = torch.zeros(6, 2, 16, 64, device=DEV), torch.zeros(6, 2, 16, 64, device=DEV)
    table = torch.tensor([[0, 1], [2, -1], [6, 5]], dtype=torch.int32, device=DEV)
    k = _normal(g, 1, 128)
    for seq, pos in [(3, 0), (2 ** 31 - 1, 0), (0, 32), (0, -1), (0, 2 ** 31 - 1), (1, 16), (2, 0)]:
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        sp = [torch.tensor([x], dtype=torch.int32, device=DEV) for x in (seq, pos)]
        paged_write(PagedCache(kp, vp), None, k, k, *sp, table, status=status)
        assert int(status) == 1 and not kp.any() and not vp.any()
        paged_write(PagedCache(kp, vp), None, k, k, *sp, table)
    paged_write(PagedCache(kp, vp), None, k, k, torch.tensor([2], dtype=torch.int32, device=DEV), torch.tensor([16], dtype=torch.int32, device=DEV),
                table, status=status.zero_())
    assert int(status) == 0 and bool(vp[5, :, 0].all())


# ---------------------------------------------------------------------------------------------------------------------
# streams, graphs, refusals
# ---------------------------------------------------------------------------------------------------------------------
def _setup(seed, dtype=torch.bfloat16, lens=(1000, 37, 0, 513)):
    g = _gen(seed)
    table, n_pages = _table(lens, 16, g)
    kp, vp = _normal(g, n_pages, 2, 16, 128, dtype=dtype), _normal(g, n_pages, 2, 16, 128, dtype=dtype)
    from paper_2406_13170_b200 import PagedCache
    return PagedCache(kp, vp), _normal(g, len(lens), 8, 128, dtype=dtype), table, torch.tensor(lens, dtype=torch.int32, device=DEV)


def test_two_streams_at_once():
    from paper_2406_13170_b200 import paged_attention
    sets = [_setup(31), _setup(32, lens=(4000, 4000, 1, 90))]
    want = [paged_attention(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(30):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(paged_attention(*sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_captured_and_replayed_beside_one_another():
    """Two graphs, each with an attention, replayed at the same time; lengths and queries change between replays."""
    from paper_2406_13170_b200 import paged_attention
    sets = [_setup(41), _setup(42, lens=(3000, 20, 777, 0))]
    graphs, outs = [], []
    for s in sets:
        paged_attention(*s)
        gr = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(gr):
            outs.append(paged_attention(*s))
        graphs.append(gr)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for step in range(4):
        for c, q, table, lens in sets:
            q.mul_(0.9)
            lens.copy_((lens - 7 * step).clamp(min=0))
        want = [paged_attention(*s) for s in sets]
        torch.cuda.synchronize()
        for _ in range(5):
            for gr, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    gr.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


LONG = [(9000, 37, 0, 30001), (20000, 1, 12345, 700)]        # many parts: through scratch


def test_two_streams_over_many_parts():
    from paper_2406_13170_b200 import paged_attention
    sets = [_setup(61, lens=LONG[0]), _setup(62, lens=LONG[1])]
    want = [paged_attention(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(30):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(paged_attention(*sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_graphs_of_several_calls_beside_one_another_and_eager_ones():
    """Calls of one capture share scratch; graphs, and the calls outside them, do not."""
    from paper_2406_13170_b200 import paged_attention
    sets = [_setup(63, lens=LONG[0]), _setup(64, lens=LONG[1])]
    graphs, outs = [], []
    for s in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append([paged_attention(*s) for _ in range(3)])
        graphs.append(gr)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for step in range(3):
        for c, q, table, lens in sets:
            q.mul_(0.9)
            lens.copy_((lens - 77 * step).clamp(min=0))
        want = [paged_attention(*s) for s in sets]
        torch.cuda.synchronize()
        eager = []
        for _ in range(4):
            for gr, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    gr.replay()
            eager.append([paged_attention(*s) for s in sets])
        torch.cuda.synchronize()
        for i, w in enumerate(want):
            assert all(torch.equal(o, w) for o in outs[i]) and all(torch.equal(e[i], w) for e in eager)


def test_empty_batches():
    from paper_2406_13170_b200 import paged_attention, paged_write
    c, q, table, lens = _setup(65)
    before = c.k_pages.clone()
    assert paged_attention(c, q[:0], table[:0], lens[:0]).shape == (0, 8, 128)
    k = torch.zeros(0, 256, device=DEV, dtype=torch.bfloat16)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    assert paged_write(c, None, k, k, none, none, table) is None
    assert paged_write(c, k.repeat(1, 4), k, k, none, none, table).shape == (0, 8, 128)
    assert torch.equal(c.k_pages, before)


def test_pages_have_to_be_aligned():
    from paper_2406_13170_b200 import AmphError, PagedCache, paged_attention
    c, q, table, lens = _setup(66)
    flat = torch.zeros(c.k_pages.numel() + 8, dtype=torch.bfloat16, device=DEV)
    odd = flat[8:].view(c.k_pages.shape)
    with pytest.raises(AmphError, match="32-byte"):
        paged_attention(PagedCache(odd, c.v_pages), q, table, lens)


def test_python_refusals():
    from paper_2406_13170_b200 import AmphError, PagedCache, paged_attention, paged_write
    c, q, table, lens = _setup(51)
    k = torch.zeros(4, 256, device=DEV, dtype=torch.bfloat16)
    seq = torch.zeros(4, dtype=torch.int32, device=DEV)
    bad = [
        lambda: paged_attention(c, q.float(), table, lens), lambda: paged_attention(c, q[:, :, :64], table, lens),
        lambda: paged_attention(c, q[:, :7].contiguous(), table, lens), lambda: paged_attention(c, q, table[:2], lens),
        lambda: paged_attention(c, q, table.long(), lens), lambda: paged_attention(c, q, table, lens[:3]),
        lambda: paged_attention(c, q, table, lens.long()), lambda: paged_attention(c, q, table, lens.cpu()),
        lambda: paged_attention(c, q, table, lens, out=q), lambda: paged_attention(c, q, table, lens, out=q.float()),
        lambda: paged_attention(c, q, table, lens, lse=torch.zeros(4, 7, device=DEV)), lambda: paged_attention(c, q.transpose(0, 1), table, lens),
        lambda: paged_attention(c, q, table, lens, scale=math.nan),
        lambda: PagedCache(c.k_pages, c.v_pages[:1]), lambda: PagedCache(c.k_pages, c.v_pages.float()),
        lambda: PagedCache(c.k_pages.transpose(1, 2), c.v_pages.transpose(1, 2)),
        lambda: PagedCache(c.k_pages[:, :, :12].contiguous(), c.v_pages[:, :, :12].contiguous()) and paged_write(
            PagedCache(c.k_pages[:, :, :12].contiguous(), c.v_pages[:, :, :12].contiguous()), None, k, k, seq, seq, table),
        lambda: paged_write(c, None, k, k.float(), seq, seq, table), lambda: paged_write(c, None, k[:, :128], k, seq, seq, table),
        lambda: paged_write(c, None, k.T, k, seq, seq, table), lambda: paged_write(c, None, k, k, seq[:3], seq, table),
        lambda: paged_write(c, None, k, k, seq, seq.long(), table), lambda: paged_write(c, None, k, k, seq, seq, table, q_out=q),
        lambda: paged_write(c, k, k, k, seq, seq, table, q_out=q), lambda: paged_write(c, None, k, k, seq, seq, table, theta=0.0),
    ]
    for call in bad:
        with pytest.raises(AmphError):
            call()
