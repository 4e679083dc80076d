"""The corners of the 8-bit paged cache: rows and masses at the ends of their ranges, calls as large as the header allows, and what the
sums' logarithms and the weights lose."""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

D = 128
U32 = 2.0 ** -24


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def vr():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    import paper_2607_15498_amd as vr
    vr.library()
    return vr


@pytest.fixture(scope="module")
def R():
    import paged8_ref
    return paged8_ref


# ---- eviction: rows of zeros beside large ones -----------------------------------------------------

@pytest.mark.parametrize("big", [3e8, 2.0 ** 20 * 448, 2.0 ** 60, 2.0 ** 127])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -118, 2.0 ** -100, 1.0])
def test_evict_zero_rows_of_large_blocks(vr, R, big, small):
    """Rows of zeros (with NaN among them, too) whose block has a large power of two, alone, beside rows of other blocks and beside the
    large row: zeros stay zeros."""
    import torch
    from test_gpu_paged8 import check_evict
    n, keep = 96, 33
    for stay in ([0, 1, 2, 3], [0, 1, 6, 40, 41], [0, 6], [0, 5, 6, 70], list(range(32)) + [40], list(range(6, 32)) + [33, 70]):
        pool = R.Pool8([n], 2, 32, 1, spare=2, fill=False, junk=0.0)
        for x in "kv":
            rows = torch.zeros((n, 2, D))
            rows[5, 0, 7] = big
            rows[6, 0, 9], rows[31, 0, 0] = math.nan, -0.0
            rows[32:64, 0, 3] = small
            rows[64:, 0] = torch.randn((32, D), generator=torch.Generator().manual_seed(3)) * small
            rows[:, 1] = torch.randn((n, D), generator=torch.Generator().manual_seed(2))
            pool.append_rows(0, 0, rows, x)
        mass = torch.zeros((1, 2, n))
        mass[0, :, stay] = 1.0
        check_evict(vr, R, [n], len(stay) if len(stay) < keep else keep, 2, 32, pool=pool, mass=mass)


# ---- eviction: as many sequences and heads as there may be -----------------------------------------

@pytest.mark.parametrize("S,G", [(65536, 64), (4100, 1024)])
def test_evict_many_heads_and_sequences(vr, S, G):
    """More (sequence, head) pairs than one launch has workgroups of this size."""
    import torch
    n, keep = 3, 2
    say(f"[evict8] S={S} G={G}")
    pages = vr.new_pages8(2, G, 32)
    for t in (pages.k, pages.v):
        t.view(torch.uint8).copy_(torch.randint(1, 120, t.shape, dtype=torch.uint8))
    before = [t.view(torch.uint8).clone() for t in (pages.k, pages.v, pages.k_scale, pages.v_scale)]
    table = torch.zeros((S, 1), dtype=torch.int32, device="cuda")
    into = torch.full((S, 1), -1, dtype=torch.int32, device="cuda")
    into[S - 1] = 1                                        # the others' rows are dropped
    mass = torch.rand((S, G, n), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    kv = (torch.arange(S, device="cuda") % (n + 1)).to(torch.int32)
    kv[S - 1] = n
    index, kept, m = vr.paged8_evict(pages, table, kv, mass, keep, into)
    k = kv.view(S, 1, 1)
    assert torch.equal(m, kv.clamp(max=keep))
    there = torch.arange(n, device="cuda") < k
    order = torch.sort(torch.where(there, mass, -1.0), dim=-1, descending=True, stable=True).indices[..., :keep]
    want = torch.sort(torch.where(torch.arange(keep, device="cuda") < k, order, n), dim=-1).values
    stay = want < n
    assert torch.equal(index, torch.where(stay, want, -1).int())
    assert torch.equal(kept, torch.where(stay, mass.gather(2, want.clamp(max=n - 1)), 0.0))
    # the last sequence's rows arrived, and their page is as it was
    for t, b in zip((pages.k, pages.v, pages.k_scale, pages.v_scale), before):
        assert torch.equal(t.view(torch.uint8)[0], b[0])
    K, V = vr.paged8_gather(pages, table[0], 32, dtype=torch.float32)
    k2, v2 = vr.paged8_gather(pages, into[S - 1], keep, dtype=torch.float32)
    for x, y in ((K, k2), (V, v2)):
        src = x.transpose(0, 1).gather(1, want[S - 1].unsqueeze(-1).expand(G, keep, D))
        assert torch.equal(y.transpose(0, 1), src)         # a smaller power holds a block's codes as they are


# ---- the logarithms of the rows' sums --------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 33), (1, 700), (7, 40), (70, 300), (1, 40000), (3, 9000), (90, 5000)])
def test_ln_sums_are_rounded_once(vr, R, dtype, m, n):
    """One key's score is far above all others' and exact in fp32, so that the logarithm is scale x score: off by its own rounding
    (half a step, 2^-24 of it), and by the exponential's and the logarithm's 2^-21.  The mass of that key is 1, off by as much."""
    import numpy as np
    import torch
    from test_gpu_paged8 import within
    G, H = 1, 4
    pool = R.Pool8([n], G, 64, seed=3, fill=False, junk=0.0)
    at = (n - m) // 2
    pool.code["v"][:] = 1.0
    pool.code["k"][int(pool.table[0, at // 64]), 0, at % 64, 9] = 320.0
    pool.exp["k"][:] = -6                                  # the key's value is 5
    gen = torch.Generator().manual_seed(n)
    q = torch.zeros((m, H, D))
    q[..., 9] = torch.exp2(4 + 6 * torch.rand((m, H), generator=gen)) + 16 * math.log(n) * 2
    q = q.to(R.tdt(dtype))
    if dtype == "f32":
        q = (q.view(torch.int32) & -4096).view(torch.float32)      # products with 5 are exact
    scale = float(np.float32(D ** -0.5))
    pages, batch = pool.device(vr), pool.batch(vr, [m])
    lse = torch.empty((m, H), device="cuda")
    vr.paged8_attn(pages, batch, q.cuda(), lse=lse)
    s = 5.0 * q[..., 9].double() * scale
    exact = s + torch.log1p((n - 1) * torch.exp(-s))
    say(f"[lse8] m={m} n={n} {dtype}: {float(s.min()):.1f} .. {float(s.max()):.1f}")
    within(lse, exact, U32 * exact * (1 + 2.0 ** -20) + 2.0 ** -21, "lse")
    got = vr.paged8_mass(pages, batch, q.cuda(), lse, torch.zeros((1, G, n), device="cuda"))[0, 0].cpu().double()
    w = torch.exp(s - exact)
    tol = float((w * (U32 * exact * (1 + 2.0 ** -20) + 2.0 ** -20)).sum())
    assert abs(float(got[at]) - float(w.sum())) <= tol + m * H * U32 * m * H, (float(got[at]) - float(w.sum()), tol)


# ---- attention mass: scores of any size ------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 5, 12, 70])
@pytest.mark.parametrize("power", [4, 10, 16, 20, 24, 28, 33, 60, 110])
def test_mass_of_large_scores(vr, R, dtype, m, power):
    """A key whose score is far above the others', up to beyond what exponents hold, is paid 1 by its row, as nearly as the logarithm
    of the row's sum says (wholly from where fp32's steps are 1 and more), and no more; the other heads' weights are what they were."""
    import torch
    n, G, H = 200, 1, 4
    pool = R.Pool8([n], G, 32, seed=m)
    for t in range(n):                                     # dim 100: one key alone
        p = int(pool.table[0, t // 32])
        pool.code["k"][p, 0, t % 32, 100] = 32.0 if t == 40 else 0.0
    q = (2.0 * torch.randn((m, H, D), generator=torch.Generator().manual_seed(1))).to(R.tdt(dtype))
    q[..., 100] = 0
    q[:, 0] = 0
    q[:, 0, 100] = 2.0 ** power
    pages, batch = pool.device(vr), pool.batch(vr, [m])
    lse = torch.empty((m, H), device="cuda")
    vr.paged8_attn(pages, batch, q.cuda(), lse=lse)
    K, _, _ = pool.rows(0)
    top = float(K[40, 0, 100]) * 2.0 ** power / math.sqrt(D)
    say(f"[mass8] m={m} {dtype} top score {top:.3g}")
    # the large row alone
    only = lse.clone()
    only[:, 1:] = -math.inf
    got = vr.paged8_mass(pages, batch, q.cuda(), only, torch.zeros((1, G, n), device="cuda"))[0, 0].cpu().double()
    assert (got >= 0).all() and (got <= (m if top >= 256 else m * (1 + 3 * U32 * top + 2.0 ** -20))).all()
    # of a row: the other keys' scores are 0.  lse is rounded once (2^-24) and so are the score's parts (2 u32), as exponents
    w = 1 / (1 + (n - 1) * math.exp(-top))
    least = 1.0 if top >= 2.0 ** 24 else w * math.exp(-3 * U32 * top) * (1 - 2.0 ** -20)
    assert got[40] >= m * least, (float(got[40]) / m, least)
    if top > 120:                                          # exp(-120) is nothing beside fp32's rounding of 1
        assert float(got.sum() - got[40]) < 1e-30
    # beside the others, which are as the reference has them
    mass = torch.rand((1, G, n), generator=torch.Generator().manual_seed(2))
    both = vr.paged8_mass(pages, batch, q.cuda(), lse, mass.cuda())[0, 0].cpu().double()
    rest = lse.cpu().clone()
    rest[:, 0] = -math.inf
    ref, tol = R.mass_ref(pool, q, [m], H, rest, mass, dtype)
    assert ((both - ref[0, 0] - got).abs() <= tol[0, 0] + 4 * (m + 2) * U32 * (ref[0, 0] + got)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 6, 70])
def test_mass_of_nan_keys(vr, R, dtype, m):
    """A NaN key that a row sees is paid NaN, which eviction puts last."""
    import torch
    n, G, H = 150, 1, 4
    pool = R.Pool8([n], G, 32, seed=m)
    for t in (17, n - 1):
        pool.code["k"][int(pool.table[0, t // 32]), 0, t % 32, 5] = math.nan
    q = torch.randn((m, H, D), generator=torch.Generator().manual_seed(1)).to(R.tdt(dtype))
    lse = torch.full((m, H), 3.0)
    got = vr.paged8_mass(pool.device(vr), pool.batch(vr, [m]), q.cuda(), lse.cuda(), torch.zeros((1, G, n), device="cuda"))[0, 0].cpu()
    assert got.isnan().nonzero()[:, 0].tolist() == [17, n - 1]


# ---- the weights of few rows -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [8, 40, 900, 9000])
@pytest.mark.parametrize("m,H", [(1, 4), (1, 16), (1, 17), (2, 9), (1, 32), (4, 8)])
def test_few_rows_keep_their_weights(vr, R, dtype, n, m, H):
    """Up to 32 rows of a KV head: what rounding takes from the weights is made good (test_paged8_weights_host.py: the bound tells),
    where a tile is whole and where it is cut, in one wave and in several."""
    from paged8_weights import case, bounds
    pool, q, live = case(n, m, H, dtype)
    out = vr.paged8_attn(pool.device(vr), pool.batch(vr, [m]), q.cuda()).cpu().double()
    ref, tol = bounds(pool, q, live, m, H, dtype)
    err = (out - ref).abs()
    say(f"[weights8] n={n} m={m} H={H} {dtype}: worst err / bound {float((err / tol).max()):.3f}")
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n", [(1, 5), (1, 3000), (70, 100), (90, 5000)])
@pytest.mark.parametrize("top", [1e30, 2.3e38, 2.6e38, 3.3e38])
def test_ln_sums_of_the_largest_scores(vr, R, dtype, m, n, top):
    """Logarithms up to the largest number, also where they pass it as powers of two: off by their own rounding (2^-24) and, there, that of
    the factor that takes one to the other (2^-23)."""
    import torch
    from test_gpu_paged8 import within
    H = 2
    pool = R.Pool8([n], 1, 32, seed=3, fill=False, junk=0.0)
    at = (n - m) // 2
    pool.code["v"][:] = 1.0
    pool.code["k"][int(pool.table[0, at // 32]), 0, at % 32, 9] = 256.0
    pool.exp["k"][:] = 0
    q = torch.zeros((m, H, D))
    q[..., 9] = top / 256
    q = q.to(R.tdt(dtype))
    lse = torch.empty((m, H), device="cuda")
    out = vr.paged8_attn(pool.device(vr), pool.batch(vr, [m]), q.cuda(), lse=lse, scale=1.0)
    exact = 256 * q[..., 9].double()
    within(lse, exact, 4 * U32 * exact, "lse")
    assert (out == 32).all()                               # a value is 1 x 2^5
    got = vr.paged8_mass(pool.device(vr), pool.batch(vr, [m]), q.cuda(), lse, torch.zeros((1, 1, n), device="cuda"), scale=1.0)[0, 0]
    assert float(got[at]) == m * H and float(got.sum()) == m * H


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 12, 30, 70])
@pytest.mark.parametrize("power", [22, 30, 60])
def test_mass_of_large_scores_of_all_dims(vr, R, dtype, m, power):
    """Scores of 2^24 and more that all 128 dims add up to: every row pays its largest key 1, and no key more."""
    import torch
    n, H = 300, 2
    pool = R.Pool8([n], 1, 32, seed=m)
    q = (2.0 ** power * torch.randn((m, H, D), generator=torch.Generator().manual_seed(power))).to(R.tdt(dtype))
    pages, batch = pool.device(vr), pool.batch(vr, [m])
    lse = torch.empty((m, H), device="cuda")
    vr.paged8_attn(pages, batch, q.cuda(), lse=lse, scale=16.0)
    assert float(lse.abs().min()) >= 2.0 ** 24
    got = vr.paged8_mass(pages, batch, q.cuda(), lse, torch.zeros((1, 1, n), device="cuda"), scale=16.0)[0, 0].cpu().double()
    K, _, _ = pool.rows(0)
    sc = torch.einsum("mhd,td->mht", q.double(), K[:, 0])
    sc = sc.masked_fill(torch.arange(n)[None, None] > torch.arange(n - m, n)[:, None, None], -math.inf)
    top, best = sc.max(-1)
    near = sc >= top[..., None] - 2.0 ** -18 * top.abs()[..., None]        # those that rounding may not tell from it
    assert (got <= near.sum((0, 1)).double()).all()
    least = torch.zeros(n, dtype=torch.float64).index_add_(0, best.flatten(), (near.sum(-1) == 1).double().flatten())
    assert (got >= least).all() and float(least.sum()) > 0.9 * m * H
