"""project_adapters on each of the ways a call can go, at sizes that take it (the kernels that ran are looked at): data that the kernel right
ahead wrote, whatever lies where no row looks, graphs whose inputs change."""
import json
import os
import subprocess
import sys

import pytest
import torch

from tests.test_gpu_adapters import DEV, _cap, _definition, _ints

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# rows, n_seg, out, in, rank, adapters, dtype, kernels of the call
PATHS = {
    "few": (5, 1, 4096, 4096, 16, 2, torch.bfloat16, ["tc_gemm_kernel", "adapter_few_kernel"]),
    "few_rank_32": (3, 1, 2048, 4096, 32, 2, torch.bfloat16, ["tc_gemm_kernel", "adapter_few_kernel"]),
    "few_rank_8": (16, 1, 4096, 4096, 8, 3, torch.bfloat16, ["tc_gemm_kernel", "adapter_few_kernel"]),
    "up": (50, 3, 2048, 2048, 16, 5, torch.bfloat16, ["tc_gemm_kernel", "adapter_down_kernel", "adapter_up_kernel"]),
    "up_rank_64": (37, 1, 4096, 4096, 64, 7, torch.bfloat16, ["tc_gemm_kernel", "adapter_down_kernel", "adapter_up_kernel"]),
    "pair": (200, 1, 2048, 2048, 32, 6, torch.bfloat16, ["tc_wide_kernel", "adapter_down_kernel", "adapter_up_kernel"]),
    "pair_512": (512, 2, 2048, 2048, 16, 40, torch.bfloat16, ["tc_wide_kernel", "adapter_down_kernel", "adapter_up_kernel"]),
    "whole": (30, 1, 512, 512, 16, 4, torch.bfloat16, ["adapter_down_kernel", "adapter_whole_kernel"]),
    "fp32": (19, 1, 512, 512, 8, 5, torch.float32, ["adapter_down_plain_kernel", "gemm_generic_kernel"]),
}
paths = pytest.mark.parametrize("path", list(PATHS))


def _ran(call):
    """Names of the kernels of a call, each once, in the order of their first launch."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    names = []
    for e in sorted(prof.events(), key=lambda e: e.time_range.start):
        name = next((n for n in ("tc_gemm_kernel", "tc_wide_kernel", "adapter_few_kernel", "adapter_down_kernel", "adapter_up_kernel",
                                 "adapter_whole_kernel", "adapter_down_plain_kernel", "gemm_generic_kernel") if n in e.name), None)
        if name and name not in names:
            names.append(name)
    return names


@pytest.fixture(scope="module")
def kernels():
    """Kernels of a call of each path.  In a process of its own: a test that counts a replayed graph's kernels was given too few of them behind a
    profiler's runs in the same process (seen once, in a run of all tests)."""
    r = subprocess.run([sys.executable, "-m", "tests.test_gpu_adapters_paths"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


class Call:
    """Whole numbers whose every partial sum fits 24 bits (and 16 bits for the low-rank products): outputs are exact, whatever the order."""

    def __init__(self, path, seed=1):
        from paper_2406_13170_b200 import Adapters
        self.rows, self.n_seg, self.out, self.in_, self.rank, self.n, self.dtype, self.kernels = PATHS[path]
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.tc = self.dtype is torch.bfloat16
        self.x, self.w, self.a, self.b, self.scale, self.at = self.inputs()
        self.ad = Adapters(self.a, self.b, self.scale)

    def inputs(self):
        g, d = self.g, self.dtype
        x = _ints(g, -1, 1, _cap(self.rows), self.in_, dtype=d)
        w = [_ints(g, -2, 2, self.out, self.in_, dtype=d) for _ in range(self.n_seg)]
        a, b = _ints(g, -1, 1, self.n, self.n_seg, self.rank, self.in_, dtype=d), _ints(g, -2, 2, self.n, self.n_seg, self.out, self.rank, dtype=d)
        scale = 2.0 ** _ints(g, -1, 2, self.n, dtype=torch.float32)
        at = torch.randint(-1, self.n, (self.rows,), generator=g, device=DEV).to(torch.int32)
        return x, w, a, b, scale, at

    def run(self, **kw):
        from paper_2406_13170_b200 import project_adapters
        return project_adapters(self.x, self.w, self.rows, self.tc, self.ad, self.at, **{"y_dtype": torch.float32, **kw})

    def want(self, x=None, w=None, a=None, b=None, scale=None, at=None):
        y = _definition(*(mine if given is None else given for mine, given in ((self.x, x), (self.w, w), (self.a, a), (self.b, b), (self.scale, scale))),
                        (self.at if at is None else at).tolist())
        assert float(y.abs().max()) < 2 ** 23
        return y.float()


@paths
def test_kernels_and_sums(path, kernels):
    c = Call(path)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert torch.equal(c.run(status=status), c.want()) and int(status) == 0
    if c.tc:
        assert torch.equal(c.run(y_dtype=torch.bfloat16), c.want().bfloat16())
    if not any(kernels.values()):
        pytest.skip("the profiler records no kernels here")
    assert kernels[path] == c.kernels


@paths
@pytest.mark.parametrize("last", ["x", "row_adapter", "a", "b", "scale", "w"])
def test_what_the_kernel_right_ahead_wrote(path, last):
    """Inputs change in place, in buffers that an earlier call has read, and nothing waits: `last` is written by the kernel ahead of the call."""
    c = Call(path)
    live = {"x": c.x, "row_adapter": c.at, "a": c.a, "b": c.b, "scale": c.scale, "w": c.w[0]}
    sets = []
    for _ in range(3):
        x, w, a, b, scale, at = c.inputs()
        sets.append({"x": x, "row_adapter": at, "a": a, "b": b, "scale": scale, "w": w[0]})
    want = [c.want(s["x"], [s["w"]] + c.w[1:], s["a"], s["b"], s["scale"], s["row_adapter"]) for s in sets]
    got = []
    torch.cuda.synchronize()
    for i in range(18):
        for name in [n for n in live if n != last] + [last]:
            torch.mul(sets[i % 3][name], 1, out=live[name])
        got.append(c.run())
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 3]), i


@pytest.mark.parametrize("path", [p for p, c in PATHS.items() if c[1] == 1 and c[2] == c[3]])
def test_a_call_s_output_is_the_next_one_s_rows(path):
    """Calls one behind another between two buffers: y is the next call's x, with nothing in between."""
    from paper_2406_13170_b200 import project_adapters
    c = Call(path)
    kind = torch.bfloat16 if c.tc else torch.float32
    w = [torch.empty_like(c.w[0]).normal_(0.0, c.in_ ** -0.5, generator=c.g)]
    c.b.mul_(c.in_ ** -0.5 / 16)
    rows = [torch.zeros_like(c.x) for _ in range(2)]

    def chain(pause):
        rows[0].copy_(c.x)
        out = []
        for i in range(24):
            project_adapters(rows[i % 2], w, c.rows, c.tc, c.ad, c.at, y=rows[1 - i % 2][: c.rows], y_dtype=kind)
            if pause:
                torch.cuda.synchronize()
                out.append(rows[1 - i % 2].clone())
                torch.cuda.synchronize()
        return out or rows[0].clone()

    slow = chain(True)
    assert torch.isfinite(slow[-1].float()).all() and slow[-1].any()
    for _ in range(4):
        assert torch.equal(chain(False), slow[-1])
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        end = chain(False)
    for _ in range(3):
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(end, slow[-1])


@pytest.mark.parametrize("path", [p for p, c in PATHS.items() if c[6] is torch.bfloat16 and c[2] == c[3]])
def test_a_call_s_output_is_the_next_one_s_weights(path):
    """512 rows times a matrix give the next call's matrix, in a buffer that has been weights before."""
    from paper_2406_13170_b200 import Adapters, project_adapters
    c = Call(path)
    d = c.in_
    m, rows = torch.zeros(d, d, dtype=torch.bfloat16, device=DEV), min(512, d)
    one = Adapters(torch.zeros(1, 1, 8, d, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 1, d, 8, dtype=torch.bfloat16, device=DEV))
    none = torch.zeros(rows, dtype=torch.int32, device=DEV)
    eye = [torch.eye(d, dtype=torch.bfloat16, device=DEV)]
    full = [_ints(c.g, -2, 2, rows, d, dtype=torch.bfloat16) for _ in range(3)]
    full = [torch.cat([f, torch.zeros(-f.shape[0] % 128, d, dtype=torch.bfloat16, device=DEV)]) for f in full]
    want = []
    for f in full:
        m[:rows].copy_(f[:rows])
        want.append(c.want(w=[m] * c.n_seg))
    torch.cuda.synchronize()
    for i in range(12):
        project_adapters(full[i % 3], eye, rows, True, one, none, y=m[:rows])
        y = project_adapters(c.x, [m] * c.n_seg, c.rows, True, c.ad, c.at, y_dtype=torch.float32)
        assert torch.equal(y, want[i % 3]), i


def test_an_attention_s_output_is_the_next_projection_s_rows():
    """The output projection of a decoding step, straight behind paged_attention, in a buffer that is used again at every step."""
    from paper_2406_13170_b200 import PagedCache, paged_attention, project_adapters
    for path in ("few", "up_rank_64"):
        c = Call(path)
        heads, dh, page = c.in_ // 128, 128, 16
        lens = torch.tensor([(37 * s) % 300 for s in range(c.rows)], dtype=torch.int32, device=DEV)
        table = torch.randperm(c.rows * 20, generator=c.g, device=DEV).to(torch.int32).view(c.rows, 20)
        kp, vp = (torch.empty(c.rows * 20, 4, page, dh, dtype=torch.bfloat16, device=DEV).normal_(generator=c.g) for _ in range(2))
        cache, x = PagedCache(kp, vp), torch.zeros_like(c.x)
        q = [torch.empty(c.rows, heads, dh, dtype=torch.bfloat16, device=DEV).normal_(generator=c.g) for _ in range(3)]

        def step(i, pause):
            paged_attention(cache, q[i % 3], table, lens, out=x[: c.rows].view(c.rows, heads, dh))
            if pause:
                torch.cuda.synchronize()
            return project_adapters(x, c.w, c.rows, True, c.ad, c.at)

        want = []
        for i in range(3):
            want.append(step(i, True))
            torch.cuda.synchronize()
        assert not torch.equal(want[0], want[1])
        got = [step(i, False) for i in range(24)]
        torch.cuda.synchronize()
        assert all(torch.equal(y, want[i % 3]) for i, y in enumerate(got))


@paths
@pytest.mark.parametrize("which", ["mixed", "runs", "one", "none"])
def test_rows_of_every_kind(path, which):
    """Rows behind the last, adapters that no row names and the scratch hold NaN and infinities; rows of y behind the last are left alone."""
    c = Call(path, seed=2)
    c.x[c.rows:] = float("nan")
    spare = c.n - 1                                    # named by no row
    rows = torch.arange(c.rows, device=DEV)
    c.at.copy_({"mixed": (rows * 7 + rows // 3) % (spare + 1) - 1, "runs": rows * spare // c.rows, "one": rows * 0 + spare - 1, "none": rows * 0 - 1}[which])
    want = c.want()
    c.a[spare], c.b[spare], c.scale[spare] = float("nan"), float("inf"), float("nan")
    junk = [torch.full((1 << 24,), float("nan"), device=DEV) for _ in range(4)]
    del junk                                           # the scratch is likely to be one of these
    buf = torch.full((c.rows + 3, c.n_seg * c.out), 7.0, device=DEV)
    c.run(y=buf[: c.rows])
    assert torch.equal(buf[: c.rows], want) and bool((buf[c.rows:] == 7.0).all())


@paths
def test_a_row_s_own_nan_is_its_own(path):
    c = Call(path, seed=3)
    c.at.copy_(torch.arange(c.rows, device=DEV) % c.n)
    y = c.run()
    c.x[1, 5] = float("nan")
    z = c.run()
    others = torch.arange(c.rows, device=DEV) != 1
    assert torch.isnan(z[1]).all() and torch.equal(z[others], y[others])
    c.x[1, 5] = 0
    mine, theirs = (c.at == 0), (c.at != 0)
    y = c.run()
    c.a[0, 0, 3, 7] = float("nan")
    z = c.run()
    assert torch.isnan(z[mine][:, : c.out]).all() and torch.equal(z[theirs], y[theirs]) and torch.equal(z[:, c.out:], y[:, c.out:])


@paths
def test_adapters_that_do_not_exist(path):
    c = Call(path, seed=4)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for wrong in (c.n, 2 ** 31 - 1):
        for row in (0, c.rows // 2, c.rows - 1):
            at = (torch.arange(c.rows, device=DEV, dtype=torch.int32) % (c.n + 1) - 1)
            at[row] = wrong
            c.at.copy_(at)
            y = c.run(status=status.zero_())
            assert int(status) == 1
            c.at[row] = -1
            assert torch.equal(y, c.want())
            assert torch.equal(c.run(status=status.zero_()), y) and int(status) == 0


@paths
def test_replays_with_other_inputs(path):
    c = Call(path, seed=5)
    c.run()
    gr = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(gr):
        y = c.run()
    for _ in range(3):
        for old, new in zip((c.x, *c.w, c.a, c.b, c.scale, c.at), (lambda x, w, *rest: (x, *w, *rest))(*c.inputs())):
            old.copy_(new)
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, c.want())


@pytest.mark.parametrize("path", [p for p in PATHS if p != "fp32"])
def test_infinite_weights_of_an_adapter(path):
    """b = inf: where the low-rank product is not zero the sum is infinite or NaN (its two bf16 halves may differ in sign), elsewhere as without it."""
    c = Call(path, seed=6)
    c.at.copy_(torch.arange(c.rows, device=DEV) % c.n)
    y = c.run()
    c.b[0, 0, 9, 2] = float("inf")
    z = c.run()
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[c.at == 0, 9] = True
    assert not torch.isfinite(z[hit]).any() and torch.equal(z[~hit], y[~hit])


if __name__ == "__main__":
    print(json.dumps({p: _ran(Call(p).run) for p in PATHS}))
