"""Low-rank adapters beside a shared projection, through the binding, against the fp64 oracle (oracle/adapt.py).

Tolerances.  A sum of n products in fp32 is off by at most (n + 2) 2^-24 (twice that: the matrix cores' own sums) of the sum of
the products' magnitudes; where blocks are summed first, n is the longest chain of additions.  bf16: operands are exact, inner
enters out, and dinner dx, as two bf16 parts (2^-17 of it is left), dinner and inner enter the gradients as three (2^-26).  (A
number x of 1 <= x < 2: the first part is off by at most half a step, 2^-8; what is left is below 2^-8, or is it and exact, where half
a step is 2^-9 2^-8 = 2^-17; what is then left is below 2^-17, where half a step is 2^-18 2^-8 = 2^-26.)  What an operand is off
by goes through the product it enters.  Outputs are rounded once: eps / 2 of their type."""
import numpy as np
import pytest
import torch

from oracle import adapt as A
from paper_1502_00512_amd import binding

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step
F32 = 2.0 ** -24


def place(a, dtype, pad=0, fill=float("nan")):
    """An array on the GPU, pad elements of NaN between its rows; and its values as the type holds them."""
    buf = torch.full((*a.shape[:-1], a.shape[-1] + pad), fill, dtype=DTYPES[dtype], device="cuda")
    buf[..., : a.shape[-1]] = torch.as_tensor(a)
    d = buf[..., : a.shape[-1]]
    return d, d.float().cpu().numpy().astype(np.float64)


def near(got, want, tol, what):
    got = got.float().cpu().numpy().astype(np.float64)
    want, tol = np.broadcast_arrays(want, tol)
    assert np.all(np.isfinite(got)), what
    off = np.abs(got - want)
    assert np.all(off <= tol), (what, np.argwhere(off > tol)[:4], np.max(off / np.maximum(tol, 1e-300)))


class Case:
    def __init__(self, M, K, N, n, R, dtype, seed=0, pad=0, ids=None, scale=True):
        rng = np.random.default_rng(seed)
        self.M, self.K, self.N, self.n, self.R, self.dtype = M, K, N, n, R, dtype
        self.x, self.X = place(rng.normal(size=(M, K)), dtype, pad)
        self.down, self.DOWN = place(rng.normal(size=(n, R, K)) / np.sqrt(K), dtype)
        self.up, self.UP = place(rng.normal(size=(n, N, R)), dtype)
        self.base, self.BASE = place(rng.normal(size=(M, N)) * 2, dtype, pad)
        self.dout, self.DOUT = place(rng.normal(size=(M, N)), dtype, pad)
        self.IDS = (rng.integers(-1, n, M) if ids is None else np.asarray(ids)).astype(np.int32)
        self.ids = torch.as_tensor(self.IDS).cuda()
        self.scale = torch.as_tensor(rng.uniform(0.5, 2.0, n).astype(np.float32)).cuda() if scale else None
        self.SCALE = np.ones(n) if self.scale is None else self.scale.cpu().numpy().astype(np.float64)
        self.rng = rng
        self.has = (self.IDS >= 0) & (self.IDS < n)
        self.of = np.where(self.has, self.IDS, 0)

    def inner_tol(self):
        size = np.einsum("mk,mrk->mr", np.abs(self.X), np.abs(self.DOWN[self.of])) * self.has[:, None]
        return 2 * (self.K + 2) * F32 * size

    def check_forward(self, with_base=True, in_place=False, **kw):
        want, INNER = A.adapter_forward(self.X, self.DOWN, self.UP, self.IDS, self.SCALE, self.BASE if with_base else None)
        base = self.base if with_base else None
        out, inner = binding.rnnlm_adapter_forward(self.x, self.down, self.up, self.ids, self.scale, base=base, out=base if in_place else None, **kw)
        di = self.inner_tol()
        near(inner, INNER, di, "inner")
        assert not inner[torch.as_tensor(~self.has).cuda()].any()
        f = (self.SCALE[self.of] * self.has)[:, None]
        size = f * np.einsum("mr,mnr->mn", np.abs(INNER), np.abs(self.UP[self.of]))
        moved = f * np.einsum("mr,mnr->mn", di, np.abs(self.UP[self.of]))
        parts = 2.0 ** -17 if self.dtype == "bf16" else 0.0
        b = np.abs(self.BASE) if with_base else 0.0
        tol = (moved + size * (2 * (2 * self.R + 4) * F32 + parts) + F32 * (b + size)) * 1.01
        near(out, want, tol + HALF[self.dtype] * (np.abs(want) + tol) + 1e-38, "out")
        free = torch.as_tensor(~self.has).cuda()
        if with_base:
            assert np.array_equal(out[free].float().cpu().numpy(), self.BASE[~self.has])
        else:
            assert not out[free].any()
        return out, inner

    def check_backward(self, with_dx=True, **kw):
        INNER = self.rng.normal(size=(self.M, self.R)).astype(np.float32)
        inner = torch.as_tensor(INNER).cuda()
        INNER = INNER.astype(np.float64)
        dx = torch.full_like(self.x, 7.0) if with_dx else None
        ddown = torch.full((self.n, self.R, self.K), 7.0, device="cuda")
        dup = torch.full((self.n, self.N, self.R), 7.0, device="cuda")
        got = binding.rnnlm_adapter_backward(self.dout, self.x, inner, self.down, self.up, self.ids, self.scale, ddown=ddown, dup=dup, dx=dx, **kw)
        assert got[0] is ddown and got[1] is dup
        DD, DU, DX = A.adapter_backward(self.DOUT, self.X, INNER, self.DOWN, self.UP, self.IDS, self.SCALE)
        a = [np.abs(t) for t in (self.DOUT, self.X, INNER, self.DOWN, self.UP)]
        rows = np.bincount(self.of[self.has], minlength=self.n)[:, None, None]
        parts = 2.0 ** -26 if self.dtype == "bf16" else 0.0
        SD, SU, SX = A.adapter_backward(*a, self.IDS, self.SCALE)  # of the magnitudes
        near(dup, DU, (2 * (rows + 4) * F32 + parts) * SU * 1.01, "dup")
        assert not dup[torch.as_tensor(rows[:, 0, 0] == 0).cuda()].any()
        chain = 140 + 8 + self.N // 512 + 1  # of dinner: a wave's columns, the waves, the blocks
        near(ddown, DD, (2 * (rows + 4 + chain) * F32 + parts) * SD * 1.01, "ddown")
        assert not ddown[torch.as_tensor(rows[:, 0, 0] == 0).cuda()].any()
        if with_dx:
            own = (2 * (2 * self.R + 4 + chain) * F32 + (2.0 ** -17 if self.dtype == "bf16" else 0.0)) * SX * 1.01
            near(dx, DX, own + HALF[self.dtype] * (np.abs(DX) + own) + 1e-38, "dx")
            assert not dx[torch.as_tensor(~self.has).cuda()].any()
        return ddown, dup, dx


BOTH = pytest.mark.parametrize("dtype", ["fp32", "bf16"])


@BOTH
@pytest.mark.parametrize("R", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 24, 31, 32, 33, 40, 48, 49, 63, 64])
def test_ranks(R, dtype):
    c = Case(70, 96, 150, 3, R, dtype, R)
    c.check_forward()
    c.check_backward()


@BOTH
@pytest.mark.parametrize("K,N", [(1, 1), (2, 3), (7, 63), (8, 64), (9, 65), (31, 127), (33, 129), (64, 255), (100, 513), (250, 1025), (257, 2049), (1000, 700),
                                 (2500, 100), (64, 10007)])
def test_widths(K, N, dtype):
    c = Case(45, K, N, 4, 6, dtype, K + N, pad=3)
    c.check_forward()
    c.check_backward()


@BOTH
@pytest.mark.parametrize("M,n", [(1, 1), (1, 5), (2, 1), (31, 40), (32, 2), (33, 1), (64, 64), (97, 3), (128, 128), (129, 1), (129, 200), (160, 7), (500, 2), (1000, 37),
                                 (3000, 1), (5000, 3)])
def test_rows_and_adapters(M, n, dtype):
    c = Case(M, 40, 90, n, 8, dtype, M + n)
    c.check_forward()
    c.check_backward()


@BOTH
@pytest.mark.parametrize("which", ["none", "one", "last", "alternating", "sorted", "falling", "most of one"])
def test_orders_of_adapters(which, dtype):
    M, n = 300, 9
    m = np.arange(M)
    ids = dict(none=np.full(M, -1), one=np.full(M, 4), last=np.full(M, n - 1), alternating=m % n, sorted=m * n // M, falling=n - 1 - m * n // M)
    ids["most of one"] = np.where(m % 50 == 0, m // 50, 8)
    c = Case(M, 33, 100, n, 10, dtype, 5, ids=ids[which])
    c.check_forward()
    c.check_backward()


@BOTH
def test_chunks_that_split_adapters(dtype):
    """Few columns and many rows: an adapter's rows lie in many chunks, and chunks hold many adapters."""
    for M, n, seed in ((2100, 1, 1), (2100, 5, 2), (1500, 400, 3), (4100, 30, 4)):
        rng = np.random.default_rng(seed)
        c = Case(M, 20, 30, n, 4, dtype, seed, ids=np.sort(rng.zipf(1.3, M) % (n + 1)) - 1)
        c.check_backward()
        c.check_forward()


@BOTH
def test_a_step_of_many_texts(dtype):
    c = Case(128, 1024, 1000, 128, 16, dtype, 3, ids=np.random.default_rng(1).permutation(128))
    c.check_forward()
    c.check_forward(with_base=False)
    c.check_forward(in_place=True)


@BOTH
def test_without_base_scale_and_dx(dtype):
    c = Case(200, 50, 70, 3, 5, dtype, 8, scale=False, pad=1)
    c.check_forward(with_base=False)
    c.check_backward(with_dx=False)


@BOTH
def test_wide_windows(dtype):
    c = Case(160, 512, 33278, 5, 16, dtype, 9)
    c.check_forward()
    c.check_backward()


@BOTH
def test_in_place_and_surroundings(dtype):
    M, N, pad = 77, 130, 13
    c = Case(M, 30, N, 4, 9, dtype, 10, pad=pad)
    out = torch.full((M + 2, N + pad), 5.0, dtype=DTYPES[dtype], device="cuda")
    got, _ = binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, c.scale, base=c.base, out=out[1: M + 1, 4: 4 + N])
    rest = out.clone()
    rest[1: M + 1, 4: 4 + N] = 5.0
    assert bool((rest == 5.0).all())
    want = got.clone()
    whole = c.base.clone()
    c.check_forward(in_place=True)
    assert torch.equal(c.base, want) and not torch.equal(whole, want)
    wide = c.base.as_strided((M, N + pad), (N + pad, 1))
    assert bool(wide[:, N:].isnan().all())


@BOTH
def test_ids_out_of_range(dtype):
    ids = np.array([0, 3, -7, 2, 1 << 30, 1, -(1 << 31), 2])
    c = Case(8, 12, 20, 3, 2, dtype, 11, ids=ids)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.check_forward(range_flag=flag)
    assert flag.item() == 1
    flag.zero_()
    c.check_backward(range_flag=flag)
    assert flag.item() == 1
    flag.zero_()
    d = Case(300, 12, 20, 3, 2, dtype, 11, ids=np.where(np.arange(300) == 299, 3, -1))
    d.check_forward(range_flag=flag)
    assert flag.item() == 1
    flag.zero_()
    Case(300, 12, 20, 3, 2, dtype, 11).check_forward(range_flag=flag)
    assert flag.item() == 0


@BOTH
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_weights_that_are_not_finite_stay_with_their_adapter(bad, dtype):
    M = 200
    c = Case(M, 24, 80, 5, 12, dtype, 12)
    want, _ = c.check_forward()
    want = want.clone()
    INNER = torch.randn(M, 12, device="cuda")
    g = binding.rnnlm_adapter_backward(c.dout, c.x, INNER, c.down, c.up, c.ids, c.scale, dx=(dx := torch.empty_like(c.x)))
    c.up[2] = bad
    c.down[3] = bad
    c.x[c.ids == 1] = bad
    free = torch.as_tensor((c.IDS != 2) & (c.IDS != 3) & (c.IDS != 1)).cuda()
    got, _ = binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, c.scale, base=c.base)
    assert torch.equal(got[free], want[free]) and not bool(got[c.ids == 2].isfinite().any())
    h = binding.rnnlm_adapter_backward(c.dout, c.x, INNER, c.down, c.up, c.ids, c.scale, dx=(dx2 := torch.empty_like(c.x)))
    for i in (0, 4):
        assert torch.equal(h[0][i], g[0][i]) and torch.equal(h[1][i], g[1][i])
    assert torch.equal(dx2[free], dx[free])


@BOTH
@pytest.mark.parametrize("N", [20, 50, 100, 200, 1100])
@pytest.mark.parametrize("R", [6, 20, 60])
def test_infinities_of_dout_are_those_of_the_formula(N, R, dtype):
    """An adapter a row, one element of each row infinite: in the first columns, in the last ones, and where the last blocks of
    columns and those in front of them share some.  (All other numbers positive, so that every sum has its infinity's sign.)"""
    M = 40
    c = Case(M, 30, N, M, R, dtype, N + R, ids=np.arange(M))
    for t, a in ((c.x, c.X), (c.down, c.DOWN), (c.up, c.UP), (c.dout, c.DOUT)):
        t.abs_()
        np.abs(a, out=a)
    column = np.unique(np.concatenate([np.arange(0, N, max(1, N // 12)), np.arange(N - 12, N), np.arange(max(0, N - 70), N, 5)]))[-M:]
    for m, v in enumerate(column):
        c.DOUT[m, v] = np.inf if m % 2 else -np.inf
        c.dout[m, int(v)] = c.DOUT[m, v]
    INNER = np.abs(c.rng.normal(size=(M, R))).astype(np.float32)
    dx = torch.empty_like(c.x)
    ddown, dup = binding.rnnlm_adapter_backward(c.dout, c.x, torch.as_tensor(INNER).cuda(), c.down, c.up, c.ids, c.scale, dx=dx)
    DD, DU, DX = A.adapter_backward(c.DOUT, c.X, INNER.astype(np.float64), c.DOWN, c.UP, c.IDS, c.SCALE)
    some = len(column)
    assert np.isinf(DD[:some]).all() and np.isinf(DX[:some]).all() and np.isfinite(DD[some:]).all()
    for got, want in ((ddown, DD), (dx, DX)):
        got = got.float().cpu().numpy()
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and np.isfinite(got[np.isfinite(want)]).all()
    got = dup.cpu().numpy()
    if dtype == "fp32":
        assert np.array_equal(got[np.isinf(DU)], DU[np.isinf(DU)])
    assert not np.isfinite(got[np.isinf(DU)]).any()  # (bf16: inner goes in as parts, of which some are zero or negative)
    assert np.isfinite(got[np.isfinite(DU)]).all()


@BOTH
def test_the_same_call_gives_the_same_bits(dtype):
    c = Case(700, 130, 3000, 11, 20, dtype, 13)
    inner = torch.randn(700, 20, device="cuda")
    first = None
    for fill in (0, 255, 77):
        ws = torch.full((binding.rnnlm_adapter_workspace_bytes(700, 130, 3000, 11, 20, int(dtype == "bf16"), True),), fill, dtype=torch.uint8, device="cuda")
        dx = torch.empty_like(c.x)
        r = (*binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, c.scale, base=c.base, workspace=ws),
             *binding.rnnlm_adapter_backward(c.dout, c.x, inner, c.down, c.up, c.ids, c.scale, dx=dx, workspace=ws), dx)
        first = r if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(r, first))


def test_no_rows():
    c = Case(0, 12, 20, 3, 2, "fp32", 14, ids=np.zeros(0))
    out, inner = binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, base=c.base)
    assert out.shape == (0, 20) and inner.shape == (0, 2)
    ddown, dup = torch.ones(3, 2, 12, device="cuda"), torch.ones(3, 20, 2, device="cuda")
    binding.rnnlm_adapter_backward(c.dout, c.x, inner, c.down, c.up, c.ids, ddown=ddown, dup=dup, dx=torch.empty_like(c.x))
    assert not ddown.any() and not dup.any()


@BOTH
def test_captured_calls_replay(dtype):
    c = Case(260, 64, 900, 6, 16, dtype, 15)
    inner, out = torch.empty(260, 16, device="cuda"), torch.empty(260, 900, dtype=DTYPES[dtype], device="cuda")
    ddown, dup, dx = torch.empty(6, 16, 64, device="cuda"), torch.empty(6, 900, 16, device="cuda"), torch.empty_like(c.x)
    ws = torch.empty(binding.rnnlm_adapter_workspace_bytes(260, 64, 900, 6, 16, int(dtype == "bf16"), True), dtype=torch.uint8, device="cuda")

    def calls():
        binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, c.scale, base=c.base, out=out, inner=inner, workspace=ws)
        binding.rnnlm_adapter_backward(c.dout, c.x, inner, c.down, c.up, c.ids, c.scale, ddown=ddown, dup=dup, dx=dx, workspace=ws)
    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        c.ids.copy_(torch.roll(c.ids, 7))  # (other adapters for the same rows: the graph reads them anew)
        calls()
        want = [t.clone() for t in (out, inner, ddown, dup, dx)]
        for t in (out, inner, ddown, dup, dx):
            t.fill_(3.0)
        ws.fill_(i * 50)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, inner, ddown, dup, dx), want))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, c.scale, base=c.base, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got[0], want[0])


@BOTH
@pytest.mark.parametrize("M,K,N,n,R", [(1 << 17, 1, 1, 1 << 16, 1), (3, 1 << 16, 1, 1, 64), (2, 1, 1 << 20, 1, 3)])
def test_largest_sizes(M, K, N, n, R, dtype):
    c = Case(M, K, N, n, R, dtype, 16)
    c.check_forward()
    c.check_backward()


def test_rows_far_apart():
    """Rows whose distance times their number passes 2^31."""
    c = Case(40, 24, 90, 3, 5, "bf16", 17)
    out, inner = binding.rnnlm_adapter_forward(c.x, c.down, c.up, c.ids, c.scale, base=c.base)
    dx = torch.empty_like(c.x)
    ddown, dup = binding.rnnlm_adapter_backward(c.dout, c.x, inner, c.down, c.up, c.ids, c.scale, dx=dx)

    def far(t=None, width=0):
        rows = torch.empty(40, 60_000_000, dtype=torch.bfloat16, device="cuda")
        assert rows.numel() > 1 << 31
        rows = rows[:, 17: 17 + (width if t is None else t.shape[1])]
        return rows if t is None else rows.copy_(t)
    x, out2 = far(c.x), far(width=90)
    got = binding.rnnlm_adapter_forward(x, c.down, c.up, c.ids, c.scale, base=far(c.base), out=out2)
    assert torch.equal(got[0], out) and torch.equal(got[1], inner)
    dx2 = far(width=24)
    got = binding.rnnlm_adapter_backward(far(c.dout), x, inner, c.down, c.up, c.ids, c.scale, dx=dx2)
    assert torch.equal(got[0], ddown) and torch.equal(got[1], dup) and torch.equal(dx2, dx)


def test_adapters_of_more_than_two_to_the_31_numbers():
    """The last of many wide adapters has what it has by itself."""
    n, N, K, R, M = 36, 1 << 20, 40, 64, 5
    gen = torch.Generator(device="cuda").manual_seed(4)
    normal = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    x, down, up, base, dout = normal(M, K), normal(n, R, K), normal(n, N, R), normal(M, N), normal(M, N)
    assert up.numel() > 1 << 31
    ids = torch.tensor([n - 1, 0, n - 1, -1, n - 1], dtype=torch.int32, device="cuda")
    out, inner = binding.rnnlm_adapter_forward(x, down, up, ids, base=base)
    dx = torch.empty_like(x)
    ddown, dup = binding.rnnlm_adapter_backward(dout, x, inner, down, up, ids, dx=dx)
    one = torch.where(ids == 0, 0, torch.where(ids < 0, -1, 1)).int()
    down2, up2 = down[[0, n - 1]].contiguous(), up[[0, n - 1]].contiguous()
    out2, inner2 = binding.rnnlm_adapter_forward(x, down2, up2, one, base=base)
    dx2 = torch.empty_like(x)
    ddown2, dup2 = binding.rnnlm_adapter_backward(dout, x, inner, down2, up2, one, dx=dx2)
    assert torch.equal(out, out2) and torch.equal(inner, inner2) and torch.equal(dx, dx2)
    assert torch.equal(ddown[[0, n - 1]], ddown2) and torch.equal(dup[0], dup2[0]) and torch.equal(dup[n - 1], dup2[1])
    assert not ddown[1: n - 1].any() and not dup[1: n - 1].any()
    want = base[0].double() + up[n - 1].double() @ inner[0].double()
    size = base[0].double().abs() + up[n - 1].double().abs() @ inner[0].double().abs()
    off = (out[0].double() - want).abs()
    own = size * (2 * (2 * R + 4) * F32 + 2.0 ** -17) * 1.01
    assert bool((off <= own + HALF["bf16"] * (want.abs() + own)).all())
