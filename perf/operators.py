"""Operators for decoding many requests over one set of weights, and the calls whose speed is tracked.

  adapters   project_adapters: a projection that all rows share and each row's own low-rank adapter beside it,
                 y[r] = x[r] . W^T + scale[a_r] * (x[r] . A[a_r]^T) . B[a_r]^T          (a_r < 0: no adapter)
  write      paged_write: rotary embedding of queries and keys at the rows' positions; keys and values go to the pages of
             their sequences (head [page][kv head][slot][head_dim]), queries come back
  attend     paged_attention: one new token of every sequence against the sequence's pages,
                 out[s][h] = softmax(q[s][h] . K[s][kv(h)]^T / sqrt(head_dim)) . V[s][kv(h)], keys 0 .. len[s] - 1

A case is a dict of plain values.  Widths, head counts, contexts and batch sizes are those of the shape table and of the
benchmark's sweep (7B, 13B and 33B widths, the two small shapes), and grouped key / value heads of the same widths.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
THETA = 10000.0


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _adapters(rows, n_seg, out, in_, rank, n_adapters, bare=0, shuffled=True, dtype="bf16", name=None):
    """rows: activation rows; bare: rows of them without an adapter; shuffled: rows of one adapter are not neighbours."""
    c = dict(kind="adapters", dtype=dtype, rows=rows, n_seg=n_seg, out=out, inp=in_, rank=rank, n_adapters=n_adapters, bare=bare,
             shuffled=shuffled)
    return dict(c, name=name) if name else c


def _write(seqs, new_lo, new_hi, past_lo, past_hi, heads, kv_heads, head_dim, page, pad=0, dtype="bf16", source="bf16", name=None):
    """Every sequence has past_lo .. past_hi tokens and gets new_lo .. new_hi more; pad: rows behind the last sequence."""
    c = dict(kind="write", dtype=dtype, source=source, seqs=seqs, new_lo=new_lo, new_hi=new_hi, past_lo=past_lo, past_hi=past_hi,
             heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, pad=pad)
    return dict(c, name=name) if name else c


def _attend(seqs, len_lo, len_hi, heads, kv_heads, head_dim, page, idle=0, dtype="bf16", name=None):
    """Sequences of len_lo .. len_hi tokens; idle: sequences of length zero among them (empty places of the batch)."""
    c = dict(kind="attend", dtype=dtype, seqs=seqs, len_lo=len_lo, len_hi=len_hi, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
             page=page, idle=idle)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request with an adapter of its own: the output projection of one token
        _adapters(1, 1, 4096, 4096, 16, 4, name="adapters_one_token"),
        # 64 requests of 24 tenants, some without an adapter: the q / k / v projection of one decoding step
        _adapters(64, 3, 4096, 4096, 16, 24, bare=5, name="adapters_qkv_64"),
        # the gate / up projection of an odd batch, adapters of a higher rank
        _adapters(37, 2, 11008, 4096, 64, 7, name="adapters_gate_up_37"),
        # a chunk of prompts of three tenants, row by row behind one another: the down projection
        _adapters(512, 1, 4096, 11008, 32, 3, shuffled=False, name="adapters_prompt_512"),
        # the small fp32 shape
        _adapters(19, 2, 688, 256, 8, 5, bare=2, dtype="fp32", name="adapters_small_fp32"),
        # one decoding step of eight sequences, fp32 rows as the projection leaves them
        _write(8, 1, 1, 300, 2000, 32, 32, 128, 16, source="fp32", name="write_step_8"),
        # one decoding step of a larger batch with grouped heads, places of the batch empty
        _write(61, 1, 1, 10, 8000, 32, 8, 128, 64, pad=3, name="write_step_61_grouped"),
        # prompts of a few sequences, one of them continued far behind its beginning
        _write(5, 700, 2600, 0, 90000, 32, 8, 128, 16, name="write_prompts"),
        # one user behind a prompt: the 7B shape
        _attend(1, 640, 640, 32, 32, 128, 16, name="attend_one_7b"),
        # eight conversations of the 13B shape's heads
        _attend(8, 90, 2048, 40, 40, 128, 64, name="attend_batch8_13b"),
        # a full server: ragged sequences, grouped heads, empty places
        _attend(64, 1, 8192, 32, 8, 128, 16, idle=3, name="attend_batch64_grouped"),
        # one very long document
        _attend(1, 131071, 131071, 32, 8, 128, 32, name="attend_document"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["adapters", "adapters", "write", "attend", "attend"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    if kind == "adapters":
        if dtype == "fp32":
            out, in_ = rng.choice([(256, 256), (688, 256), (256, 688), (1000, 256)])
            rows = _log_int(rng, 1, 100)
        else:
            out, in_ = rng.choice([(4096, 4096), (11008, 4096), (4096, 11008), (5120, 5120), (13824, 5120), (6656, 6656),
                                   (512, 512), (1408, 512), (512, 1408), (1000, 520)])
            rows = _log_int(rng, 1, 512)
        n_seg = rng.randint(1, 3) if out * in_ <= 27e6 else 1
        while n_seg > 1 and rows * n_seg * out * in_ > 512 * 45e6:
            n_seg -= 1
        if rows * n_seg * out * in_ > 512 * 45e6:
            rows = 300
        return _adapters(rows, n_seg, out, in_, rng.choice([8, 16, 16, 24, 32, 64]), _log_int(rng, 1, 32),
                         bare=rng.randint(0, rows // 3), shuffled=rng.random() < 0.6, dtype=dtype)
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    heads = kv_heads * (1 if kv_heads == 32 else rng.choice([1, 2, 4, 5, 8]))
    page = rng.choice([1, 8, 16, 16, 32, 64, 256])
    per_token = 2 * kv_heads * head_dim * (4 if dtype == "fp32" else 2)
    if kind == "write":
        seqs = _log_int(rng, 1, 64)
        past = _log_int(rng, 1, 60000 // seqs + 1)
        if rng.random() < 0.5:
            lo = hi = 1
        else:
            hi = max(2, int(min(4000, 7000 / seqs)))
            hi = _log_int(rng, 2, hi)
            lo = max(1, hi // 3)
        return _write(seqs, lo, hi, past // 2, past, heads, kv_heads, head_dim, page, pad=rng.choice([0, 0, 3]), dtype=dtype,
                      source=rng.choice(["bf16", "fp32"]))
    most = 4.8e8 / per_token if dtype == "bf16" else 1e8 / per_token
    seqs = _log_int(rng, 1, 96)
    hi = _log_int(rng, 16, max(17, min(120000, 2 * most / seqs)))
    return _attend(seqs, max(1, hi // rng.choice([2, 8, 64])), hi, heads, kv_heads, head_dim, page,
                   idle=rng.randint(0, seqs // 8), dtype=dtype)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _plain_random(case):
    """Lengths, row orders: from the case alone, so that work() knows them."""
    return random.Random("/".join("%s=%s" % (k, v) for k, v in sorted(case.items()) if k != "name"))


def _row_adapters(case):
    rng = _plain_random(case)
    rows, n = case["rows"], case["n_adapters"]
    idx = [-1] * min(case["bare"], rows - 1)
    idx += [i * n // (rows - len(idx)) if rows - len(idx) >= n else rng.randrange(n) for i in range(rows - len(idx))]
    if case["shuffled"]:
        rng.shuffle(idx)
    return idx


def _lengths(case, n, lo, hi):
    rng = _plain_random(case)
    v = [lo + int((hi - lo) * rng.random() ** 1.5) for _ in range(n)]
    v[rng.randrange(n)] = hi
    return v


def _write_rows(case):
    """(tokens behind which each sequence goes on, new tokens of each)"""
    past = _lengths(case, case["seqs"], case["past_lo"], case["past_hi"])
    new = _lengths(dict(case, kind="new"), case["seqs"], case["new_lo"], case["new_hi"])
    return past, new


def _attend_lengths(case):
    v = _lengths(case, case["seqs"], case["len_lo"], case["len_hi"])
    rng = _plain_random(dict(case, kind="idle"))
    longest = max(range(len(v)), key=lambda i: v[i])
    for i in rng.sample([i for i in range(len(v)) if i != longest], min(case["idle"], len(v) - 1)):
        v[i] = 0
    return v


def _page_table(lengths, page, gen):
    """Pages in random places; entries behind a sequence's last page hold what an allocator leaves there (-1)."""
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + max(2, sum(need) // 16)
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    width = max(1, max(need))
    first = torch.tensor([0] + need, device=DEVICE).cumsum(0)[:-1]
    at = first[:, None] + torch.arange(width, device=DEVICE)[None]
    inside = torch.arange(width, device=DEVICE)[None] < torch.tensor(need, device=DEVICE)[:, None]
    table = torch.where(inside, order[at.clamp(max=n_pages - 1)], torch.full_like(order[:1], -1))
    return table.contiguous(), n_pages


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed * 2654435761 % (1 << 40) + 17)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=DEVICE).normal_(0.0, std, generator=gen)

    if case["kind"] == "adapters":
        rows, n_seg, out, in_, rank, n = (case[k] for k in ("rows", "n_seg", "out", "inp", "rank", "n_adapters"))
        cap = -(-rows // 16) * 16 if rows <= 128 else -(-rows // 128) * 128
        st = dict(case=case, rows=rows, x=normal(cap, in_), w=[normal(out, in_, std=0.02) for _ in range(n_seg)],
                  a=normal(n, n_seg, rank, in_, std=in_ ** -0.5), b=normal(n, n_seg, out, rank, std=0.02 * (in_ / rank) ** 0.5 / 4),
                  scale=torch.rand(n, generator=gen, device=DEVICE) * 1.5 + 0.5,
                  row_adapter=torch.tensor(_row_adapters(case), dtype=torch.int32, device=DEVICE))
        if own:
            from paper_2406_13170_b200 import Adapters
            st["adapters"] = Adapters(st["a"], st["b"], st["scale"])
        return st
    heads, kv, dh, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    if case["kind"] == "write":
        past, new = _write_rows(case)
        table, n_pages = _page_table([p + n for p, n in zip(past, new)], page, gen)
        seq = [s for s, n in enumerate(new) for _ in range(n)] + [-1] * case["pad"]
        pos = [p + i for p, n in zip(past, new) for i in range(n)] + [0] * case["pad"]
        # what an earlier projection left: queries, keys and values of a row behind one another
        qkv = normal(len(seq), (heads + 2 * kv) * dh, dtype=DTYPES[case["source"]])
        st = dict(case=case, q=qkv[:, : heads * dh], k=qkv[:, heads * dh: (heads + kv) * dh], v=qkv[:, (heads + kv) * dh:],
                  row_seq=torch.tensor(seq, dtype=torch.int32, device=DEVICE), row_pos=torch.tensor(pos, dtype=torch.int32, device=DEVICE),
                  table=table, k_pages=normal(n_pages, kv, page, dh), v_pages=normal(n_pages, kv, page, dh),
                  q_out=torch.zeros(len(seq), heads, dh, dtype=dt, device=DEVICE))
    else:
        lengths = _attend_lengths(case)
        table, n_pages = _page_table(lengths, page, gen)
        st = dict(case=case, q=normal(len(lengths), heads, dh, std=1.5), lens=torch.tensor(lengths, dtype=torch.int32, device=DEVICE),
                  table=table, k_pages=normal(n_pages, kv, page, dh), v_pages=normal(n_pages, kv, page, dh))
    if own:
        from paper_2406_13170_b200 import PagedCache
        st["cache"] = PagedCache(st["k_pages"], st["v_pages"])
    return st


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _plain_adapters(st):
    """Every adapter's low-rank product for every row, those of other adapters set to zero."""
    rows, (n, n_seg, rank, _) = st["rows"], st["a"].shape
    x = st["x"][:rows].float()
    at = st["row_adapter"].long()
    mine = (at[:, None] == torch.arange(n, device=at.device)[None]).float() * st["scale"][None]                     # [rows, n]
    t = torch.einsum("ri,nsji->rnsj", x, st["a"].float()) * mine[:, :, None, None]
    low = torch.einsum("rnsj,nsoj->rso", t, st["b"].float())
    base = torch.stack([x @ w.float().T for w in st["w"]], dim=1)
    return (base + low).reshape(rows, -1).to(st["x"].dtype)


def _plain_write(st):
    case = st["case"]
    dh, page = case["head_dim"], case["page"]
    keep = (st["row_seq"] >= 0).nonzero()[:, 0]
    seq, pos = st["row_seq"][keep].long(), st["row_pos"][keep].long()
    freq = THETA ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=pos.device) / dh)
    ang = pos.double()[:, None] * freq[None]
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def rotated(x):
        x = x[keep].float().reshape(len(keep), -1, dh)
        lo, hi = x[..., : dh // 2], x[..., dh // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)

    pages, slots = st["table"][seq, pos // page].long(), pos % page
    st["q_out"][keep] = rotated(st["q"]).to(st["q_out"].dtype)
    st["k_pages"][pages, :, slots] = rotated(st["k"]).to(st["k_pages"].dtype)
    st["v_pages"][pages, :, slots] = st["v"][keep].reshape(len(keep), -1, dh).to(st["v_pages"].dtype)
    return st["q_out"], st["k_pages"], st["v_pages"]


def _plain_attend(st):
    q, lens, table = st["q"].float(), st["lens"].long(), st["table"].long()
    seqs, heads, dh = q.shape
    _, kv, page, _ = st["k_pages"].shape
    width = table.shape[1] * page
    inside = torch.arange(width, device=q.device)[None] < lens[:, None]                                              # [seqs, keys]
    table = table.clamp(min=0)
    k = st["k_pages"][table].float().permute(0, 2, 1, 3, 4).reshape(seqs, kv, width, dh)
    s = q.reshape(seqs, kv, heads // kv, dh) @ k.transpose(2, 3) / math.sqrt(dh)
    del k
    s = torch.where(inside[:, None, None], s, torch.full_like(s[:1, :1, :1, :1], -math.inf))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    v = st["v_pages"][table].float().permute(0, 2, 1, 3, 4).reshape(seqs, kv, width, dh)
    v = torch.where(inside[:, None, :, None], v, torch.zeros_like(v[:1, :1, :1, :1]))
    o = p @ v / torch.where(total == 0, torch.ones_like(total), total)
    return o.reshape(seqs, heads, dh).to(st["q"].dtype)


def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2406_13170_b200 import paged_attention, paged_write, project_adapters
        if kind == "adapters":
            covered = st["case"]["dtype"] == "bf16" and st["case"]["out"] % 128 == 0 and st["case"]["inp"] % 64 == 0
            return project_adapters(st["x"], st["w"], st["rows"], covered, st["adapters"], st["row_adapter"])
        if kind == "write":
            q = paged_write(st["cache"], st["q"], st["k"], st["v"], st["row_seq"], st["row_pos"], st["table"], theta=THETA, q_out=st["q_out"])
            return q, st["k_pages"], st["v_pages"]
        return paged_attention(st["cache"], st["q"], st["table"], st["lens"])
    return {"adapters": _plain_adapters, "write": _plain_write, "attend": _plain_attend}[kind](st)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    esz = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "adapters":
        rows, n_seg, out, in_, rank = (case[k] for k in ("rows", "n_seg", "out", "inp", "rank"))
        idx = _row_adapters(case)
        used, served = len(set(i for i in idx if i >= 0)), sum(i >= 0 for i in idx)
        return {"bytes": esz * (rows * in_ + n_seg * out * in_ + used * n_seg * rank * (in_ + out) + rows * n_seg * out) + 4 * rows,
                "flops": 2 * n_seg * (rows * out * in_ + served * rank * (in_ + out))}
    heads, kv, dh, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    if case["kind"] == "write":
        past, new = _write_rows(case)
        rows = sum(new)
        src = 4 if case["source"] == "fp32" else 2
        return {"bytes": rows * ((heads + 2 * kv) * dh * (src + esz) + 8) + 4 * sum(-(-(p + n) // page) - p // page for p, n in zip(past, new)),
                "flops": rows * (heads + kv) * dh * 3}
    lengths = _attend_lengths(case)
    return {"bytes": sum(lengths) * 2 * kv * dh * esz + 2 * len(lengths) * heads * dh * esz + 4 * (len(lengths) + sum(-(-n // page) for n in lengths)),
            "flops": 4 * sum(lengths) * heads * dh}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "adapters":
        idx = _row_adapters(case)
        y = torch.empty(case["rows"], case["n_seg"], case["out"], dtype=torch.float64, device=DEVICE)
        for s in range(case["n_seg"]):
            w = st["w"][s].double()
            for a in sorted(set(idx)):
                at = [r for r, i in enumerate(idx) if i == a]
                m = w if a < 0 else w + float(st["scale"][a]) * (st["b"][a, s].double() @ st["a"][a, s].double())
                y[at, s] = st["x"][at].double() @ m.T
        return y.reshape(case["rows"], -1)
    dh, page, dt = case["head_dim"], case["page"], DTYPES[case["dtype"]]
    if case["kind"] == "write":
        past, new = _write_rows(case)
        q_out, k_pages, v_pages = st["q_out"].double(), st["k_pages"].double(), st["v_pages"].double()
        turn = torch.tensor([THETA ** (-2.0 * i / dh) for i in range(dh // 2)], dtype=torch.float64, device=DEVICE)
        r0 = 0
        for s, (p, n) in enumerate(zip(past, new)):
            at = torch.arange(p, p + n, device=DEVICE)
            z = torch.polar(torch.ones(n, dh // 2, dtype=torch.float64, device=DEVICE), at.double()[:, None] * turn)[:, None]
            q, k, v = (st[m][r0: r0 + n].double().reshape(n, -1, dh) for m in ("q", "k", "v"))
            q, k = (torch.complex(x[..., : dh // 2].contiguous(), x[..., dh // 2:].contiguous()) * z for x in (q, k))
            q_out[r0: r0 + n] = torch.cat([q.real, q.imag], dim=-1)
            pages = st["table"][s, at // page].long()
            k_pages[pages, :, at % page] = torch.cat([k.real, k.imag], dim=-1)
            v_pages[pages, :, at % page] = v
            r0 += n
        return q_out, k_pages, v_pages
    lengths, heads, kv = _attend_lengths(case), case["heads"], case["kv_heads"]
    o = torch.zeros(len(lengths), heads, dh, dtype=torch.float64, device=DEVICE)
    for s, n in enumerate(lengths):
        if n:
            at = torch.arange(n, device=DEVICE)
            pages = st["table"][s, at // page].long()
            k, v = (st[m][pages, :, at % page].double().transpose(0, 1) for m in ("k_pages", "v_pages"))          # [kv, n, dh]
            z = torch.einsum("hgd,hnd->hgn", st["q"][s].double().reshape(kv, heads // kv, dh), k) * dh ** -0.5
            o[s] = torch.einsum("hgn,hnd->hgd", torch.softmax(z, dim=-1), v).reshape(heads, dh)
    return o
