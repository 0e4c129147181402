"""project_adapters: the shared projection with each row's own low-rank adapter beside it, against the definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TOL = 2e-4          # the projection tests' tolerance for sums of fp32 on the tensor cores, relative to the largest output


def _cap(rows):
    return -(-rows // 16) * 16 if rows <= 128 else -(-rows // 128) * 128


def _ints(g, lo, hi, *shape, dtype):
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV).to(dtype)


def _definition(x, ws, a, b, scale, idx):
    """fp64 [rows, n_seg * out]."""
    rows, n_seg = len(idx), len(ws)
    y = torch.stack([x[:rows].double() @ w.double().T for w in ws], 1)
    for r, i in enumerate(idx):
        if 0 <= i < a.shape[0]:
            for s in range(n_seg):
                t = a[i, s].double() @ x[r].double()
                y[r, s] += (1.0 if scale is None else float(scale[i])) * (b[i, s].double() @ t)
    return y.reshape(rows, -1)


# rows, n_seg, out, in, rank, adapters, tensor cores
SHAPES = [
    (1, 1, 128, 64, 8, 1, True),
    (1, 1, 4096, 4096, 16, 4, True),
    (5, 2, 256, 128, 16, 3, True),
    (16, 3, 512, 512, 24, 5, True),
    (17, 1, 1408, 512, 128, 2, True),
    (64, 3, 512, 1408, 64, 70, True),
    (100, 8, 128, 128, 40, 9, True),
    (130, 1, 384, 512, 16, 2, True),
    (512, 2, 512, 256, 32, 3, True),
    (300, 1, 4096, 1024, 8, 300, True),
    (3, 1, 200, 72, 8, 2, False),                  # shapes that only the plain projection takes
    (19, 2, 1000, 520, 16, 4, False),
    (33, 1, 7, 8, 8, 5, False),
    (40, 3, 50, 136, 56, 6, False),
]


def _rows_of(case, rows, n):
    g = torch.Generator().manual_seed(rows)
    if case == "one":
        return [n - 1] * rows
    if case == "none":
        return [-1] * rows
    if case == "runs":
        return [min(n - 1, r * n // rows) for r in range(rows)]
    idx = torch.randint(-1, n, (rows,), generator=g).tolist()
    return [i if i >= 0 else (-1 if r % 2 else -2 ** 31) for r, i in enumerate(idx)]


@pytest.mark.parametrize("which", ["mixed", "runs", "one", "none"])
@pytest.mark.parametrize("rows,n_seg,out,in_,rank,n,tc", SHAPES)
def test_sums_of_whole_numbers(rows, n_seg, out, in_, rank, n, tc, which):
    """Whole numbers whose every partial sum fits 24 bits (and 16 bits for the low-rank products): the outputs are exact, whatever the order."""
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(rows * 7 + out)
    for dtype, y_dtype in ((torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)):
        use = tc and dtype is torch.bfloat16
        x = _ints(g, -1, 1, _cap(rows), in_, dtype=dtype)
        ws = [_ints(g, -2, 2, out, in_, dtype=dtype) for _ in range(n_seg)]
        a, b = _ints(g, -1, 1, n, n_seg, rank, in_, dtype=dtype), _ints(g, -2, 2, n, n_seg, out, rank, dtype=dtype)
        scale = 2.0 ** _ints(g, -1, 2, n, dtype=torch.float32)
        idx = _rows_of(which, rows, n)
        at = torch.tensor(idx, dtype=torch.int32, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        y = project_adapters(x, ws, rows, use, Adapters(a, b, scale), at, y_dtype=y_dtype, status=status)
        want = _definition(x, ws, a, b, scale, idx)
        assert float(want.abs().max()) < 2 ** 23
        assert int(status) == 0 and y.dtype is y_dtype
        assert torch.equal(y, want.to(torch.float32).to(y_dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,n_seg,out,in_,rank,n,tc", SHAPES)
def test_values(rows, n_seg, out, in_, rank, n, tc, dtype):
    from paper_2406_13170_b200 import Adapters, project_adapters
    if dtype is torch.float32 and rows * n_seg * out * in_ > 2e9:
        pytest.skip("the plain kernel's sizes")
    g = torch.Generator(device=DEV).manual_seed(rows + in_)

    def normal(*shape, std=1.0):
        return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(dtype)

    x, ws = normal(_cap(rows), in_), [normal(out, in_, std=0.02) for _ in range(n_seg)]
    a, b = normal(n, n_seg, rank, in_, std=in_ ** -0.5), normal(n, n_seg, out, rank, std=0.3)
    idx = _rows_of("mixed", rows, n)
    at = torch.tensor(idx, dtype=torch.int32, device=DEV)
    y = project_adapters(x, ws, rows, tc and dtype is torch.bfloat16, Adapters(a, b), at, y_dtype=torch.float32)
    want = _definition(x, ws, a, b, None, idx)
    big = max(1.0, float(want.abs().max()))
    assert float((y.double() - want).abs().max()) <= TOL * big
    again = project_adapters(x, ws, rows, tc and dtype is torch.bfloat16, Adapters(a, b), at, y_dtype=torch.float32)
    assert torch.equal(y, again)
    if dtype is torch.bfloat16:
        y = project_adapters(x, ws, rows, tc, Adapters(a, b), at)
        assert y.dtype is torch.bfloat16
        assert bool(((y.double() - want).abs() <= TOL * big + 2.0 ** -8 * want.abs()).all())


LARGE = [                                            # enough weights and rows for the tcgen05 kernels, odd tiles of both
    (1, 8, 1024, 2048, 8, 1, True),
    (5, 2, 2048, 2048, 16, 3, True),
    (3, 1, 1024, 4096, 32, 2, True),                  # up to 16 rows of a small rank: sums and adapters in one kernel
    (16, 1, 2048, 1408, 24, 4, True),
    (9, 2, 4096, 1024, 8, 9, True),
    (17, 1, 4096, 1408, 128, 2, True),
    (64, 3, 2048, 1408, 64, 70, True),
    (70, 3, 768, 1024, 8, 4, True),
    (130, 1, 1024, 2048, 16, 2, True),
    (512, 2, 1024, 512, 32, 3, True),
    (333, 3, 2560, 576, 56, 40, True),
    (300, 3, 1000, 520, 64, 20, False),
]


@pytest.mark.parametrize("which", ["mixed", "runs", "one", "none"])
@pytest.mark.parametrize("rows,n_seg,out,in_,rank,n,tc", LARGE)
def test_sums_of_whole_numbers_in_large(rows, n_seg, out, in_, rank, n, tc, which):
    test_sums_of_whole_numbers(rows, n_seg, out, in_, rank, n, tc, which)


@pytest.mark.parametrize("rows,n_seg,out,in_,rank,n,tc", LARGE)
def test_values_in_large(rows, n_seg, out, in_, rank, n, tc):
    test_values(rows, n_seg, out, in_, rank, n, tc, torch.bfloat16)


@pytest.mark.parametrize("tc", [True, False], ids=["tcgen05", "plain"])
def test_rows_do_not_meet_other_adapters(tc):
    """Adapters that no row names, and rows behind the last, may hold anything; so may the scratch."""
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(3)
    rows, out, in_, rank, n = 21, 256, 192, 16, 6
    x = torch.full((_cap(rows), in_), float("nan"), dtype=torch.bfloat16, device=DEV)
    x[:rows] = _ints(g, -1, 1, rows, in_, dtype=torch.bfloat16)
    w = _ints(g, -2, 2, out, in_, dtype=torch.bfloat16)
    a, b = _ints(g, -1, 1, n, 1, rank, in_, dtype=torch.bfloat16), _ints(g, -1, 1, n, 1, out, rank, dtype=torch.bfloat16)
    a[2], b[2], a[4] = float("nan"), float("inf"), float("inf")
    idx = [(0, 1, 3, 5, -1)[r % 5] for r in range(rows)]
    junk = [torch.full((1 << 22,), float("nan"), device=DEV) for _ in range(4)]
    del junk                                          # the scratch is likely to be one of these
    y = project_adapters(x, [w], rows, tc, Adapters(a, b), torch.tensor(idx, dtype=torch.int32, device=DEV), y_dtype=torch.float32)
    good = [0, 1, 3, 5]
    want = _definition(x, [w], torch.nan_to_num(a, 0, 0, 0), torch.nan_to_num(b, 0, 0, 0), None, idx)
    assert good and torch.equal(y.double(), want)
    # a NaN of one's own stays with one's own rows
    y2 = project_adapters(x, [w], rows, tc, Adapters(a, b), torch.tensor([2] + idx[1:], dtype=torch.int32, device=DEV), y_dtype=torch.float32)
    assert torch.isnan(y2[0]).all() and torch.equal(y2[1:], y[1:])


@pytest.mark.parametrize("tc", [True, False], ids=["tcgen05", "plain"])
def test_adapters_that_do_not_exist_are_reported(tc):
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(4)
    x, w = _ints(g, -1, 1, 16, 128, dtype=torch.bfloat16), _ints(g, -2, 2, 128, 128, dtype=torch.bfloat16)
    a, b = _ints(g, -1, 1, 2, 1, 8, 128, dtype=torch.bfloat16), _ints(g, -1, 1, 2, 1, 128, 8, dtype=torch.bfloat16)
    for wrong in (2, 2 ** 31 - 1):
        idx = [0, wrong, 1]
        at = torch.tensor(idx, dtype=torch.int32, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        y = project_adapters(x, [w], 3, tc, Adapters(a, b), at, y_dtype=torch.float32, status=status)
        assert int(status) == 1
        assert torch.equal(y.double(), _definition(x, [w], a, b, None, idx))
        project_adapters(x, [w], 3, tc, Adapters(a, b), at)


def test_side_stream_and_capture():
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(5)
    x, w = _ints(g, -1, 1, 64, 256, dtype=torch.bfloat16), [_ints(g, -2, 2, 512, 256, dtype=torch.bfloat16) for _ in range(3)]
    a, b = _ints(g, -1, 1, 4, 3, 16, 256, dtype=torch.bfloat16), _ints(g, -1, 1, 4, 3, 512, 16, dtype=torch.bfloat16)
    ad = Adapters(a, b)
    at = torch.tensor([r % 5 - 1 for r in range(50)], dtype=torch.int32, device=DEV)
    want = project_adapters(x, w, 50, True, ad, at)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        y = [project_adapters(x, w, 50, True, ad, at) for _ in range(10)]
    z = [project_adapters(x, w, 50, True, ad, at) for _ in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in y + z)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = project_adapters(x, w, 50, True, ad, at)
    x.copy_(_ints(g, -1, 1, 64, 256, dtype=torch.bfloat16))
    at.copy_((at + 2) % 4)
    w[0].neg_()
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, project_adapters(x, w, 50, True, ad, at)) and not torch.equal(out, want)


def test_two_graphs_beside_one_another():
    """Replayed at the same time on two streams, each with its own scratch; the same calls outside at the same time."""
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(8)
    sets = []
    for rows, n_seg, out, in_, rank in ((50, 3, 2048, 1024, 16), (200, 2, 1024, 2048, 32)):
        x, w = _ints(g, -1, 1, _cap(rows), in_, dtype=torch.bfloat16), [_ints(g, -2, 2, out, in_, dtype=torch.bfloat16) for _ in range(n_seg)]
        ad = Adapters(_ints(g, -1, 1, 5, n_seg, rank, in_, dtype=torch.bfloat16), _ints(g, -1, 1, 5, n_seg, out, rank, dtype=torch.bfloat16))
        at = torch.tensor([r * 7 % 6 - 1 for r in range(rows)], dtype=torch.int32, device=DEV)
        sets.append((x, w, rows, True, ad, at))
    want = [project_adapters(*s) for s in sets]
    graphs, outs = [], []
    for s in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append([project_adapters(*s) for _ in range(2)])
        graphs.append(gr)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    eager = []
    for _ in range(6):
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        eager.append([project_adapters(*s) for s in sets])
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        assert all(torch.equal(o, w) for o in outs[i]) and all(torch.equal(e[i], w) for e in eager)


def test_an_output_as_the_next_call_s_weights():
    """What a call leaves is there for the next one, whatever it takes it for."""
    from paper_2406_13170_b200 import Adapters, project_adapters
    g = torch.Generator(device=DEV).manual_seed(9)
    rows, d = 512, 512
    x, w = _ints(g, -1, 1, rows, d, dtype=torch.bfloat16), _ints(g, -1, 1, d, d, dtype=torch.bfloat16)
    ad = Adapters(_ints(g, 0, 1, 1, 1, 8, d, dtype=torch.bfloat16) * 0, _ints(g, -1, 1, 1, 1, d, 8, dtype=torch.bfloat16))
    at = torch.zeros(rows, dtype=torch.int32, device=DEV)
    for _ in range(20):
        y = project_adapters(x, [w], rows, True, ad, at)                       # [512, 512]: whole numbers below 2^8 are exact in bf16
        z = project_adapters(x, [y], rows, True, ad, at, y_dtype=torch.float32)
        want = x.double() @ (x.double() @ w.double().T).to(torch.bfloat16).double().T
        assert torch.equal(z.double(), want)
        x = x.roll(1, 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_an_empty_batch(dtype):
    """Answered as the paged operators answer it: nothing is launched."""
    from paper_2406_13170_b200 import Adapters, AmphError, project_adapters
    z = lambda *s, dt=dtype: torch.zeros(s, dtype=dt, device=DEV)                 # noqa: E731
    ad, w, none = Adapters(z(2, 3, 8, 128), z(2, 3, 256, 8)), [z(256, 128)] * 3, z(0, dt=torch.int32)
    tc = dtype is torch.bfloat16
    for x in (z(16, 128), z(0, 128)):
        y = project_adapters(x, w, 0, tc, ad, none)
        assert y.shape == (0, 768) and y.dtype is dtype and y.is_cuda
        assert project_adapters(x, w, 0, tc, ad, none, y_dtype=torch.float32).dtype is torch.float32
        y = z(0, 768)
        assert project_adapters(x, w, 0, tc, ad, none, y=y) is y
    for bad in (lambda: project_adapters(z(16, 128), w[:2], 0, tc, ad, none), lambda: project_adapters(z(16, 128), w, 0, tc, ad, z(1, dt=torch.int32)),
                lambda: project_adapters(z(16, 128), w, 0, tc, ad, none, y=z(1, 768))):
        with pytest.raises(AmphError):
            bad()


def test_any_sequence_of_weights():
    """As for `project`: a tuple, a module's list of parameters, what indexes and counts itself."""
    from paper_2406_13170_b200 import Adapters, project, project_adapters
    c = _ints(torch.Generator(device=DEV).manual_seed(10), -1, 1, 16 + 2 * 256, 128, dtype=torch.bfloat16)
    x, w = c[:16], [c[16: 272], c[272:]]
    ad = Adapters(torch.zeros(2, 2, 8, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 2, 256, 8, dtype=torch.bfloat16, device=DEV))
    at = torch.zeros(5, dtype=torch.int32, device=DEV)

    class Two:
        def __len__(self):
            return 2

        def __getitem__(self, i):
            return w[i]

    want = project_adapters(x, w, 5, True, ad, at, y_dtype=torch.float32)
    for ws in (tuple(w), torch.nn.ParameterList([torch.nn.Parameter(t, requires_grad=False) for t in w]), Two()):
        assert torch.equal(project(x, ws, 5, True), want)
        assert torch.equal(project_adapters(x, ws, 5, True, ad, at, y_dtype=torch.float32), want)


def test_python_refusals():
    from paper_2406_13170_b200 import Adapters, AmphError, project_adapters
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device=DEV)        # noqa: E731
    ad = Adapters(z(2, 1, 8, 128), z(2, 1, 256, 8))
    at = z(3, dt=torch.int32)
    x, w = z(16, 128), z(256, 128)
    project_adapters(x, [w], 3, True, ad, at)
    bad = [
        lambda: project_adapters(x, [w, w], 3, True, ad, at), lambda: project_adapters(x.float(), [w], 3, True, ad, at),
        lambda: project_adapters(x, [w.T], 3, True, ad, at), lambda: project_adapters(x, [w], 4, True, ad, at),
        lambda: project_adapters(x, [w], 3, True, ad, at.long()), lambda: project_adapters(x, [w], 3, True, ad, at.cpu()),
        lambda: project_adapters(x[:, ::2], [w], 3, True, ad, at), lambda: project_adapters(x[:8], [w], 3, True, ad, at),
        lambda: project_adapters(x, [w], 3, True, ad, at, y=z(3, 255)), lambda: project_adapters(x, [w], 3, True, ad, at, y_dtype=torch.float16),
        lambda: project_adapters(x, [w], 3, True, ad, at, y=z(3, 256), y_dtype=torch.float32),
        lambda: project_adapters(x.float(), [w.float()], 3, True, Adapters(z(2, 1, 8, 128, dt=torch.float32), z(2, 1, 256, 8, dt=torch.float32)), at),
        lambda: project_adapters(x.float(), [w.float()], 3, False, Adapters(z(2, 1, 8, 128, dt=torch.float32), z(2, 1, 256, 8, dt=torch.float32)), at,
                                 y_dtype=torch.bfloat16),
        lambda: project_adapters(x, [w], 3, True, Adapters(z(2, 1, 4, 128), z(2, 1, 256, 4)), at),
        lambda: Adapters(z(2, 1, 8, 128), z(2, 1, 256, 8), z(3, dt=torch.float32)), lambda: Adapters(z(2, 1, 8, 128), z(2, 2, 256, 8)),
        lambda: Adapters(z(0, 1, 8, 128), z(0, 1, 256, 8)),
    ]
    for call in bad:
        with pytest.raises(AmphError):
            call()
