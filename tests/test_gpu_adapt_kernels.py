"""The kernels that large calls of the operators that adapt a model take: the adapters' forward pass and gradients over wide windows and
long chunks of rows, the preference loss's rows that meet in every shape, against 64-bit products and softmaxes.  (That these sizes
take these kernels is tested without a GPU: test_adapt_kernels_cpu.py.)

Tolerances: as in test_gpu_adapters.py and test_gpu_policy.py, on the GPU."""
import pytest
import torch

import test_gpu_adapters as adapters
import test_gpu_policy as policy
from oracle import adapt as A
from paper_1502_00512_amd import binding

pytestmark = pytest.mark.gpu

DTYPES, HALF, F32 = adapters.DTYPES, adapters.HALF, adapters.F32
IN_PARTS = {"fp32": 0.0, "bf16": 1.0}  # operands in fp32 go in as bf16 numbers

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
    bf16 = IN_PARTS[dtype]
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


@pytest.mark.parametrize("dtype,M,N,R", [("bf16", 2017, 33279, 16), ("fp32", 1009, 33279, 16), ("bf16", 2017, 33279, 48), ("fp32", 1009, 33279, 32)])
def test_infinities_in_the_last_columns_of_wide_windows(dtype, M, N, R):
    """One infinite element of dout an adapter, in columns that the last wave and the one in front have in common (N = 33279: 1 to 127
    of them).  (up and down are positive, x is not zero.)"""
    K, n, dt = 40, 6, DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(R)
    normal = lambda *s, t=dt: torch.empty(*s, dtype=t, device="cuda").normal_(generator=gen)  # noqa: E731
    x, down, up, inner, dout = normal(M, K), normal(n, R, K).abs_(), normal(n, N, R).abs_(), normal(M, R, t=torch.float32), normal(M, N)
    x[x == 0], down[down == 0], up[up == 0] = 1.0, 1.0, 1.0
    ids = torch.arange(M, device="cuda", dtype=torch.int32) % n
    columns = [N - 1, N - 2, N - 31, N - 33, N - 60, N - 127]
    for a, v in enumerate(columns):
        dout[600 + a, v] = float("inf") if a % 2 else -float("inf")  # (600 % n = 0)
    dx = torch.empty_like(x)
    ddown, dup = binding.rnnlm_adapter_backward(dout, x, inner, down, up, ids, dx=dx)
    for a, v in enumerate(columns):
        d = dout[600 + a, v].float()
        assert bool((ddown[a] == d * x[600 + a].float()).all()) and bool((dx[600 + a].float() == d).all()), (a, v)
    spoilt = torch.zeros(n, N, dtype=torch.bool, device="cuda")
    spoilt[torch.arange(n, device="cuda"), torch.tensor(columns, device="cuda")] = True
    assert torch.equal(~dup.isfinite(), spoilt[..., None].expand(n, N, R))
    others = torch.ones(M, dtype=torch.bool, device="cuda")
    others[600: 600 + n] = False
    assert bool(dx[others].isfinite().all())


# T, pairs, words of bf16 (half as many of fp32), and the shape of the kernel in which they meet (None: two passes)
MEET = [
    (64, 15, 8203, (256, 6)), (64, 8, 16383, (256, 8)), (64, 5, 24001, (512, 6)), (64, 4, 32001, (512, 8)), (40, 5, 40009, (512, 12)),
    (64, 3, 64001, (512, 16)), (64, 2, 80003, (512, 20)), (50, 2, 100003, (512, 25)), (64, 1, 120007, (1024, 18)), (40, 1, 204807, (1024, 25)),
    (1, 200, 64001, (512, 16)),
    # next to them: rows of 1024 slots, texts of 65 positions, rows that no shape holds
    (64, 15, 8199, None), (65, 3, 64001, None), (40, 1, 204811, None),
]


def words(dtype, V):
    return V if dtype == "bf16" else V // 2


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,P,V,shape", MEET)
@pytest.mark.parametrize("in_place", [False, True])
def test_preference_rows_of_every_shape(T, P, V, shape, in_place, dtype):
    V = words(dtype, V)
    gen = torch.Generator(device="cuda").manual_seed(V)
    z = torch.empty(T, 2 * P, V, dtype=DTYPES[dtype], device="cuda").normal_(0.0, 2.0, generator=gen)
    y = torch.randint(0, V, (T, 2 * P), generator=gen, device="cuda", dtype=torch.int32)
    y[torch.rand(T, 2 * P, generator=gen, device="cuda") < 0.2] = -1
    y[0, 0] = -1
    Z = z.double()
    Z[0, 0] = 0.0
    z[0, 0] = float("nan")
    beta, eps, scale = 0.25, 0.125, 0.5
    has, at = y >= 0, y.long().clamp(min=0)[..., None]
    l = torch.log_softmax(Z, 2)
    q = l.exp()
    l = torch.where(has, l.gather(2, at)[..., 0], 0.0)
    share = 1.0 / has.sum(0).clamp(min=1).double()
    S = l.sum(0) * share
    ref = (S + torch.randn(2 * P, generator=gen, device="cuda")).float()
    r = S - ref.double()
    r = r[:P] - r[P:]
    soft = torch.nn.functional.softplus
    L = (1 - eps) * soft(-beta * r) + eps * soft(beta * r)
    f = beta * (torch.sigmoid(beta * r) - (1 - eps))
    f = torch.cat([f, -f]) * share * scale
    most = Z.abs().amax(2)
    terms = 26 * 8 + 1
    if shape is None:
        terms = max(terms, V // 512 + 1)
    E = torch.where(has, (terms * 1.1 + 24) * F32 + F32 * (4 * most + 2), 0.0)
    dS = E.sum(0) * share + 1e-15 * S.abs()
    dr = dS[:P] + dS[P:]
    hit = torch.zeros_like(q).scatter_(2, at, 1.0)
    want = torch.where(has[..., None], f[:, None] * (hit - q), 0.0)
    of_value = (E + F32 * (4 * most + 8))[..., None]
    F = f.abs()[:, None]
    df = (share * scale * (beta * beta / 4) * torch.cat([dr, dr]) + F32 * f.abs())[:, None]
    tol = F * (q * of_value + hit * 2 * F32) + df * (hit - q).abs() + HALF[dtype] * want.abs() * (1 + 2 * of_value) + F * 2.0 ** -100 + 2.0 ** -126
    results = []
    for polls in (256, 0):
        try:
            binding.rnnlm_set_preference_wait(polls)
            rows = z.clone()
            dz = rows if in_place else torch.full_like(z, 5.0)
            loss, logp = binding.rnnlm_preference_loss(rows, y, ref, beta=beta, smoothing=eps, mean=True, scale=scale, dlogits=dz)
            torch.cuda.synchronize()
        finally:
            binding.rnnlm_set_preference_wait(256)
        results.append((loss, logp, dz))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    loss, logp, dz = results[0]
    near(logp, S, dS + F32 * S.abs(), "logp")
    near(loss, L, (beta + beta * beta / 4 * dr) * dr + F32 * L + 1e-14 * (1 + beta * r.abs()), "loss")
    near(dz, want, tol, "dlogits")
    assert not dz[~has].any()


@pytest.mark.parametrize("dtype,T,P,V", [("bf16", 64, 3, 64001), ("fp32", 64, 1, 60003)])
def test_preference_rows_that_meet_against_the_oracle(dtype, T, P, V):
    d, z, y, rng = policy.draw_preference(T, P, V, dtype, 50)
    ref = (A.preference(z, y)[1] + rng.normal(size=2 * P)).astype("float32")
    policy.check_preference(d, z, y, ref, None, dtype, "logistic", 0.2, 0.1, in_place=True)
