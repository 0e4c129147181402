"""The operators for decoding many requests as a program uses them: an attention block of a decoding step, prompts first, then steps whose
every stage is compared with its definition in 64 bits on the stage's own inputs; captured steps against eager ones."""
import pytest
import torch

from tests.test_gpu_adapters import TOL, _cap, _definition
from tests.test_gpu_paged import DEV, HALF, _check_attention, _gen, _near, _normal, _rotated, _table

pytestmark = pytest.mark.gpu
THETA = 10000.0


class Block:
    """One attention block: q and k / v projections with adapters, rotary embedding and cache write, attention, output projection."""

    def __init__(self, dtype, d, heads, kv, dh, page, room, n_adapters, seed=5):
        from paper_2406_13170_b200 import Adapters, PagedCache
        g = _gen(seed)
        self.dtype, self.d, self.heads, self.kv, self.dh, self.page = dtype, d, heads, kv, dh, page
        self.tc = dtype is torch.bfloat16
        widths = {"q": (1, heads * dh, d), "kv": (2, kv * dh, d), "o": (1, d, heads * dh)}
        self.w, self.ab, self.ad = {}, {}, {}
        for name, (n_seg, out, in_) in widths.items():
            self.w[name] = [_normal(g, out, in_, dtype=dtype, std=in_ ** -0.5) for _ in range(n_seg)]
            a = _normal(g, n_adapters, n_seg, 16, in_, dtype=dtype, std=in_ ** -0.5)
            b = _normal(g, n_adapters, n_seg, out, 16, dtype=dtype, std=0.2)
            scale = torch.rand(n_adapters, generator=g, device=DEV) + 0.5
            self.ab[name] = (a, b, scale)
            self.ad[name] = Adapters(a, b, scale)
        self.table, n_pages = _table(room, page, g)
        self.k_pages = _normal(g, n_pages, kv, page, dh, dtype=dtype)
        self.v_pages = _normal(g, n_pages, kv, page, dh, dtype=dtype)
        self.cache = PagedCache(self.k_pages, self.v_pages)

    def project(self, name, x, rows, at):
        from paper_2406_13170_b200 import project_adapters
        return project_adapters(x, self.w[name], rows, self.tc, self.ad[name], at)

    def write(self, x, rows, at, seq, pos):
        from paper_2406_13170_b200 import paged_write
        q, kv = self.project("q", x, rows, at), self.project("kv", x, rows, at)
        half = self.kv * self.dh
        return q, kv, paged_write(self.cache, q, kv[:, :half], kv[:, half:], seq, pos, self.table, theta=THETA)

    def step(self, x, rows, at, seq, pos, lens, padded):
        """padded: [cap, heads * dh], rows behind the last are left as they are."""
        from paper_2406_13170_b200 import paged_attention
        q, kv, turned = self.write(x, rows, at, seq, pos)
        paged_attention(self.cache, turned, self.table, lens, out=padded[:rows].view(rows, self.heads, self.dh))
        return q, kv, turned, self.project("o", padded, rows, at)

    def check_projection(self, name, got, x, at):
        a, b, scale = self.ab[name]
        want = _definition(x, self.w[name], a, b, scale, at.tolist())
        big = max(1.0, float(want.abs().max()))
        assert bool(((got.double() - want).abs() <= TOL * big + HALF[self.dtype] * want.abs()).all())


PROMPTS = [70, 1, 0, 129, 33]


def _block(dtype, dh, steps):
    heads, kv = (8, 2) if dh == 64 else (4, 4)
    return Block(dtype, 512, heads, kv, dh, 16, [n + steps for n in PROMPTS], 3)


def _prompts(blk):
    n = sum(PROMPTS)
    g = _gen(77)
    x = _normal(g, _cap(n), blk.d, dtype=blk.dtype)
    seq = torch.tensor([s for s, p in enumerate(PROMPTS) for _ in range(p)], dtype=torch.int32, device=DEV)
    pos = torch.tensor([i for p in PROMPTS for i in range(p)], dtype=torch.int32, device=DEV)
    blk.write(x, n, (seq % 4 - 1).to(torch.int32), seq, pos)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_steps_of_an_attention_block(dtype, dh):
    steps, rows = 3, len(PROMPTS)
    blk = _block(dtype, dh, steps)
    _prompts(blk)
    g = _gen(78)
    seq = torch.arange(rows, dtype=torch.int32, device=DEV)
    at = torch.tensor([0, 2, -1, 0, 1], dtype=torch.int32, device=DEV)
    padded = torch.zeros(_cap(rows), blk.heads * dh, dtype=dtype, device=DEV)
    for t in range(steps):
        x = _normal(g, _cap(rows), blk.d, dtype=dtype)
        pos = torch.tensor([p + t for p in PROMPTS], dtype=torch.int32, device=DEV)
        lens = pos + 1
        q, kv, turned, out = blk.step(x, rows, at, seq, pos, lens, padded)
        blk.check_projection("q", q, x, at)
        blk.check_projection("kv", kv, x, at)
        want, size = _rotated(q, pos, blk.heads, dh, THETA)
        assert _near(turned, want, size)
        pages, slots = blk.table[seq.long(), pos.long() // 16].long(), pos.long() % 16
        want, size = _rotated(kv[:, : blk.kv * dh], pos, blk.kv, dh, THETA)
        assert _near(blk.k_pages[pages, :, slots], want, size)
        assert torch.equal(blk.v_pages[pages, :, slots], kv[:, blk.kv * dh:].reshape(rows, blk.kv, dh))
        attended = padded[:rows].view(rows, blk.heads, dh)
        from paper_2406_13170_b200 import paged_attention
        lse = torch.empty(rows, blk.heads, device=DEV)
        assert torch.equal(paged_attention(blk.cache, turned, blk.table, lens, lse=lse), attended)
        _check_attention(attended, lse, turned, blk.k_pages, blk.v_pages, blk.table, lens.tolist())
        blk.check_projection("o", out, padded, at)
    assert not padded[rows:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_captured_steps_are_the_eager_ones(dtype):
    steps, rows = 6, len(PROMPTS)
    seq = torch.arange(rows, dtype=torch.int32, device=DEV)
    at = torch.tensor([0, 2, -1, 0, 1], dtype=torch.int32, device=DEV)
    xs = [_normal(_gen(90 + t), _cap(rows), 512, dtype=dtype) for t in range(steps)]

    def start():
        blk = _block(dtype, 128, steps)
        _prompts(blk)
        return blk, torch.tensor(PROMPTS, dtype=torch.int32, device=DEV), torch.zeros(_cap(rows), blk.heads * 128, dtype=dtype, device=DEV)

    blk, pos, padded = start()
    want = []
    for x in xs:
        want.append(blk.step(x, rows, at, seq, pos, pos + 1, padded)[-1].clone())
        pos += 1
    blk, pos, padded = start()
    x = xs[0].clone()
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = blk.step(x, rows, at, seq, pos, pos + 1, padded)[-1]
        pos += 1
    for t in range(steps):
        x.copy_(xs[t])
        gr.replay()
        assert torch.equal(out, want[t])
