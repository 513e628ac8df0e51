"""The kernels that large calls of the operators that adapt a model take: the adapters' forward pass and gradients over wide windows and
long chunks of rows, against 64-bit products.  (That these sizes take these kernels is tested without a GPU:
test_adapt_kernels_cpu.py.)

Tolerances: as in test_gpu_adapters.py, on the GPU."""
import pytest
import torch

import test_gpu_adapters as adapters
from paper_1502_00512_amd import binding

pytestmark = pytest.mark.gpu

DTYPES, HALF, F32 = adapters.DTYPES, adapters.HALF, adapters.F32
POWER = {"fp32": 0.0, "bf16": 1.0}

# dtype, rows, N, n, R, and the kernel that forms dup (columns of a wave / 16, rank / 16).  Up to 2^27 bytes of dout the ranks up to
# 16 have columns of their own.
GRAD = [
    ("bf16", 2016, 33279, 5, 5, (1, 4)), ("bf16", 2017, 33279, 5, 5, (1, 8)),
    ("bf16", 2016, 33279, 3, 16, (1, 4)), ("bf16", 2017, 33279, 3, 16, (1, 8)),
    ("fp32", 1008, 33279, 5, 5, (1, 2)), ("fp32", 1009, 33279, 5, 5, (1, 4)),
    ("fp32", 1008, 33279, 3, 16, (1, 2)), ("fp32", 1009, 33279, 3, 16, (1, 4)),
    # chunks of 1024 positions, the most that one holds: few adapters, many, and one a row
    ("bf16", 2048, 131071, 4, 16, (1, 8)), ("bf16", 2048, 131071, 300, 3, (1, 8)), ("fp32", 2048, 65001, 7, 5, (1, 4)),
    ("fp32", 2048, 65001, 2048, 1, (1, 4)), ("bf16", 2048, 65001, 6, 20, (2, 4)), ("bf16", 3000, 33279, 9, 40, (3, 4)),
    ("bf16", 2048, 65001, 5, 64, (4, 4)), ("fp32", 2048, 64001, 5, 31, (2, 4)), ("fp32", 1000, 65001, 3, 40, (3, 2)),
    ("fp32", 1024, 64001, 2, 64, (4, 2)),
]


def near(got, want, tol, what):
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (what, (off - tol).max().item(), (off / tol.clamp(min=1e-300)).max().item())


@pytest.mark.parametrize("dtype,M,N,n,R,kernel", GRAD)
def test_adapters_over_wide_windows(dtype, M, N, n, R, kernel):
    K, dt = 61, DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(M + N + R)
    normal = lambda *s, t=dt: torch.empty(*s, dtype=t, device="cuda").normal_(generator=gen)  # noqa: E731
    x, down, up, inner = normal(M, K), normal(n, R, K), normal(n, N, R), normal(M, R, t=torch.float32)
    dout, base = normal(M, N), normal(M, N)
    scale = 0.5 + torch.rand(n, generator=gen, device="cuda")
    ids = torch.randint(-1 if n < M else 0, n, (M,), generator=gen, device="cuda", dtype=torch.int32)
    if n == M:
        ids = torch.randperm(M, generator=gen, device="cuda").to(torch.int32)
    ddown, dup, dx = torch.full((n, R, K), 7.0, device="cuda"), torch.full((n, N, R), 7.0, device="cuda"), torch.full_like(x, 7.0)
    binding.rnnlm_adapter_backward(dout, x, inner, down, up, ids, scale, ddown=ddown, dup=dup, dx=dx)
    out, u = binding.rnnlm_adapter_forward(x, down, up, ids, scale, base=base)
    bf16 = POWER[dtype]
    chain = 140 + 8 + N // 512 + 1  # of dinner: a wave's columns, the waves, the blocks
    for a in range(-1, n):
        rows = (ids == a).nonzero()[:, 0]
        if a < 0 or len(rows) == 0:
            assert not dx[rows].any() and not u[rows].any() and torch.equal(out[rows], base[rows])
            if a >= 0:
                assert not ddown[a].any() and not dup[a].any()
            continue
        d, X, I, f = dout[rows].double(), x[rows].double(), inner[rows].double(), scale[a].double()
        D, U = down[a].double(), up[a].double()
        g = f * (d @ U)
        size = f * (d.abs() @ U.abs())
        count = len(rows)
        near(dup[a], f * (d.T @ I), (2 * (count + 4) * F32 + bf16 * 2.0 ** -26) * f * (d.abs().T @ I.abs()) * 1.01, ("dup", a))
        near(ddown[a], g.T @ X, (2 * (count + 4 + chain) * F32 + bf16 * 2.0 ** -26) * (size.T @ X.abs()) * 1.01, ("ddown", a))
        own = (2 * (2 * R + 4 + chain) * F32 + bf16 * 2.0 ** -17) * (size @ D.abs()) * 1.01
        want = g @ D
        near(dx[rows], want, own + HALF[dtype] * (want.abs() + own) + 1e-38, ("dx", a))
        V = X @ D.T
        dv = 2 * (K + 2) * F32 * (X.abs() @ D.abs().T)
        near(u[rows], V, dv, ("inner", a))
        b = base[rows].double()
        want, size = b + f * (V @ U.T), f * (V.abs() @ U.abs().T)
        own = (f * (dv @ U.abs().T) + size * (2 * (2 * R + 4) * F32 + bf16 * 2.0 ** -17) + F32 * (b.abs() + size)) * 1.01
        near(out[rows], want, own + HALF[dtype] * (want.abs() + own) + 1e-38, ("out", a))
