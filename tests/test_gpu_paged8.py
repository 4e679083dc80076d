"""GPU parity of the 8-bit paged cache (append, attention, attention mass, eviction, gather) against plain implementations
in 64 bits on the host (paged8_ref.py, which derives the bounds).  Codes, scales, eviction and gather are exact."""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

D, B = 128, 32


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


def within(got, ref, tol, what):
    got = got.detach().cpu().double()
    both = got.isnan() & ref.isnan() | (got == ref)
    err = (got - ref).abs()
    bad = ~((err <= tol) | both)
    worst = float((err / tol.clamp_min(1e-300)).masked_fill(both, 0.0).nan_to_num(0.0).max()) if err.numel() else 0.0
    say(f"  {what}: worst err / bound {worst:.3f}")
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {worst}, at {bad.nonzero()[:4].tolist()}"


# ---- append and gather ---------------------------------------------------------------------------

def new_rows(R, n, G, dtype, gen):
    import torch
    x = torch.randn((n, G, D), generator=gen) * torch.exp2(torch.randint(-3, 4, (n, G, 1), generator=gen))
    return x.to(R.tdt(dtype))


def check_append(vr, R, calls, G, page, dtype, fused=False, seed=0, pad=0, junk=math.nan):
    """calls: for each call, every sequence's new tokens; all lengths add up."""
    import torch
    total = [sum(c[s] for c in calls) for s in range(len(calls[0]))]
    say(f"[append8] calls {calls if len(calls) < 5 else len(calls)} G={G} page={page} {dtype} fused={fused}")
    pool = R.Pool8(total, G, page, seed, junk=junk, fill=False)
    pages = pool.device(vr)
    gen = torch.Generator().manual_seed(seed + 1)
    at = [0] * len(total)
    for q_len in calls:
        T = sum(q_len) + 2 * pad
        k, v = (new_rows(R, T, G, dtype, gen) for _ in range(2))
        i = pad
        for s, m in enumerate(q_len):
            pool.append_rows(s, at[s], k[i:i + m], "k")
            pool.append_rows(s, at[s], v[i:i + m], "v")
            at[s] += m
            i += m
        pool.kv_len = list(at)
        kd, vd = k.cuda(), v.cuda()
        if fused:
            x = torch.zeros((T, 2 * G + 3, D), dtype=k.dtype, device="cuda")
            x[:, 1:1 + G], x[:, G + 2:2 * G + 2] = kd, vd
            kd, vd = x[:, 1:1 + G], x[:, G + 2:2 * G + 2]
        vr.paged8_append(pages, pool.batch(vr, q_len, pad), kd, vd)
    torch.cuda.synchronize()
    pool.same(pages)
    return pool, pages


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 100, 257])
def test_append_prompt(vr, R, dtype, n):
    check_append(vr, R, [[n]], 2, 32 if n % 2 else 64, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_append_ragged_calls(vr, R, dtype, page):
    """Chunks, single tokens and nothing, call after call: blocks are left half full and their scales rise."""
    check_append(vr, R, [[5, 0, 40, 1], [1, 3, 0, 1], [70, 1, 1, 33], [1, 1, 1, 1], [2, 90, 31, 0]], 3, page, dtype, seed=page, pad=page // 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_token_by_token(vr, R, dtype):
    check_append(vr, R, [[1, 1]] * 70, 1, 32, dtype, fused=True, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_many_rows(vr, R, dtype):
    """More rows than waves take one by one: chunks that begin and end inside blocks, and many single tokens."""
    check_append(vr, R, [[17, 9], [2100, 300], [1, 77]], 4, 128, dtype, fused=True, seed=4, pad=3)
    check_append(vr, R, [[1] * 300, [1] * 300], 32, 32, dtype, seed=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_extremes(vr, R, dtype):
    """Zeros, the smallest and the largest numbers, infinities and NaN, both sides of 448, ties, and a scale that takes what was
    there to zero."""
    import torch
    pool = R.Pool8([32 * 9], 1, 32, 0, fill=False, junk=0.0)
    pages = pool.device(vr)
    x = torch.zeros((32 * 9, 1, D))
    x[32:64, 0, 3] = -0.0
    x[64, 0, :6] = torch.tensor([448.0, 449.0, -447.0, 0.0009765625, 0.00146484375, 2.0 ** -9])
    x[96:98, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 7.0])
    x[128, 0, :3] = torch.tensor([3.3e38, -2.9e38, 1e30])
    x[160, 0, :4] = torch.tensor([1e-38, -3e-37, 1e-33, 2.0 ** -110])
    x[192:224, 0] = math.nan
    ties = torch.arange(128).float()                       # halves between codes of 8 .. 15.5, and of 16 .. 31
    x[224, 0] = 8 + ties / 16
    x[225, 0] = 16 + ties / 8
    x[225, 0, 0] = 448.0
    x[256, 0, :5] = torch.tensor([224.0, 1.75, 256.0, 448.0, 1.0])
    x = x.to(R.tdt(dtype))
    kv = torch.tensor([32 * 9], dtype=torch.int32).cuda()
    vr.paged8_append(pages, pool.batch(vr, [32 * 9]), x.cuda(), (2 * x).cuda())
    pool.append_rows(0, 0, x, "k")
    pool.append_rows(0, 0, 2 * x, "v")
    pool.same(pages)
    # one row at a time into one block: 1, then 2^40, then infinity, then 2^119 x 1.9
    pool = R.Pool8([4], 1, 32, 0, fill=False, junk=0.0)
    pages = pool.device(vr)
    for i, y in enumerate((1.0, 2.0 ** 40, math.inf, 1.9 * 2.0 ** 119)):
        row = torch.full((1, 1, D), y).to(R.tdt(dtype))
        row[0, 0, 5] = math.nan
        pool.kv_len = [i + 1]
        vr.paged8_append(pages, pool.batch(vr, [1]), row.cuda(), row.cuda())
        for name in "kv":
            pool.append_rows(0, i, row, name)
        pool.same(pages)


@pytest.mark.parametrize("many", [False, True])
def test_append_bad_entries(vr, R, many):
    """Bad pages drop their rows, lengths outside the table and negative positions too; nothing else is written."""
    import torch
    n = 1100 if many else 130
    pool = R.Pool8([n, n, 40, 40], 8, 32, 1, width=(n + 31) // 32, fill=False)
    for i, bad in ((0, -1), (2, pool.total), (3, -(1 << 31)), (4, (1 << 31) - 1)):
        pool.table[0, i] = bad
    pages = pool.device(vr)
    lens = [n, n + 100000, -3, 25]                          # beyond the table; negative; 15 of 40 rows before position 0
    q_len = [n, 50, 40, 40]
    gen = torch.Generator().manual_seed(2)
    k, v = (new_rows(R, sum(q_len), 8, "bf16", gen) for _ in range(2))
    for x, rows in (("k", k), ("v", v)):
        pool.append_rows(0, 0, rows[:n], x)
        pool.append_rows(3, 0, rows[-25:], x)
    pool.kv_len = lens
    vr.paged8_append(pages, pool.batch(vr, q_len), k.cuda(), v.cuda())
    pool.same(pages)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 700])
def test_gather(vr, R, dtype, n):
    import torch
    pool = R.Pool8([max(n, 1)], 3, 64, n)
    if n > 200:
        pool.table[0, 1], pool.table[0, 2] = -1, pool.total
    pages = pool.device(vr)
    K, V = vr.paged8_gather(pages, pool.table[0].cuda(), n, dtype=R.tdt(dtype))
    k, v, ok = pool.rows(0, n)
    for got, want in ((K, k), (V, v)):
        want = torch.where(ok[:, None, None], want, 0.0).to(R.tdt(dtype))
        assert got.shape == (n, 3, D) and got.dtype == R.tdt(dtype) and torch.equal(got.cpu(), want)


# ---- attention -----------------------------------------------------------------------------------

def check_attn(vr, R, q_len, kv_len, G, H, page, dtype, causal=True, window=0, seed=0, pool=None, scale=None, qscale=2.0, lse=True):
    import torch
    say(f"[attn8] q {q_len} kv {kv_len} G={G} H={H} page={page} {dtype} causal={causal} window={window}")
    pool = pool or R.Pool8(kv_len, G, page, seed)
    T = sum(q_len)
    q = (qscale * torch.randn((T, H, D), generator=torch.Generator().manual_seed(seed + 1))).to(R.tdt(dtype))
    pages, batch = pool.device(vr), pool.batch(vr, q_len)
    z = torch.full((T, H), 7.0, dtype=torch.float32, device="cuda") if lse else None
    out = vr.paged8_attn(pages, batch, q.cuda(), causal=causal, window=window, scale=scale, lse=z)
    torch.cuda.synchronize()
    ref, tol, lref, ltol = R.attn_ref(pool, q, q_len, H, dtype, causal, window, scale)
    within(out, ref, tol, "out")
    if lse:
        within(z, lref, ltol, "lse")
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 511, 513, 2100])
def test_attn_single_token(vr, R, dtype, n):
    check_attn(vr, R, [1], [n], 2, 8, 32, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 16, 31, 33, 64, 65, 100, 130, 257])
def test_attn_prompt(vr, R, dtype, n):
    check_attn(vr, R, [n], [n], 1, 3, 32, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,H,page", [(1, 2, 32), (4, 28, 64), (8, 32, 256), (3, 3, 128), (1, 40, 32)])
def test_attn_ragged_batch(vr, R, dtype, G, H, page):
    """Chunks, prompts, single tokens and sequences with nothing new or nothing at all, together."""
    check_attn(vr, R, [1, 0, 40, 7, 1, 0, 3], [300, 50, 170, 7, 1, 0, 1000], G, H, page, dtype, seed=H)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([1, 1, 2], [1500, 40, 700]), ([60], [1700]), ([130, 5], [900, 1100])])
@pytest.mark.parametrize("window", [1, 16, 63, 64, 65, 500])
def test_attn_window(vr, R, dtype, q_len, kv_len, window):
    check_attn(vr, R, q_len, kv_len, 2, 4, 32, dtype, window=window, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([1], [700]), ([5, 2], [33, 2000]), ([70], [300]), ([150], [40])])
def test_attn_all_keys(vr, R, dtype, q_len, kv_len):
    check_attn(vr, R, q_len, kv_len, 2, 6, 32, dtype, causal=False, seed=kv_len[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([3, 9], [1, 0]), ([40, 2], [17, 1])])
def test_attn_rows_that_see_nothing(vr, R, dtype, q_len, kv_len):
    """More new tokens than the cache holds: the first ones stand before it and get zeros, and -infinity for their sums."""
    out = check_attn(vr, R, q_len, kv_len, 2, 4, 32, dtype, seed=9)
    assert (out[:q_len[0] - kv_len[0]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_many_sequences(vr, R, dtype):
    kv = [1 + (37 * s) % 211 for s in range(150)]
    check_attn(vr, R, [1] * 150, kv, 1, 2, 32, dtype, seed=4)
    check_attn(vr, R, [min(k, 1 + s % 50) for s, k in enumerate(kv)], kv, 1, 2, 32, dtype, seed=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [[1, 1], [6, 8], [90, 30]])
def test_attn_large_scores(vr, R, dtype, q_len):
    """Logits in the hundreds, of both signs, and one far above: the maximum moves late and by far; and tiny ones."""
    pool = R.Pool8([900, 333], 2, 64, seed=6)
    p, at = int(pool.table[0, 13]), 850 % 64
    pool.exp["k"][p, :, at // 32] += 3
    check_attn(vr, R, q_len, [900, 333], 2, 8, 64, dtype, pool=pool, seed=6, qscale=20.0)
    check_attn(vr, R, q_len, [900, 333], 2, 8, 64, dtype, pool=pool, seed=6, scale=1e-3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [[1, 4], [60, 45]])
def test_attn_bad_pages(vr, R, dtype, q_len):
    """Entries that name no page: their tokens are left out (a sequence of bad pages alone: zeros)."""
    pool = R.Pool8([700, 500], 2, 32, seed=8)
    for i, bad in ((0, -1), (3, pool.total), (4, -(1 << 31)), (9, (1 << 31) - 1), (21, pool.total + 7)):
        pool.table[0, i] = bad
    check_attn(vr, R, q_len, [700, 500], 2, 8, 32, dtype, pool=pool, seed=8)
    pool.table[1] = -1
    out = check_attn(vr, R, q_len, [700, 500], 2, 8, 32, dtype, pool=pool, seed=8)
    assert (out[q_len[0]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,window", [([50], 0), ([3], 0), ([50], 20), ([3], 20), ([12], 5)])
def test_attn_nan_values(vr, R, dtype, q_len, window):
    """NaN among values reach the rows that see them and no others; NaN keys of later tokens reach nobody."""
    n = 90
    pool = R.Pool8([n], 1, 32, seed=q_len[0])
    for t, dim in ((2, 5), (60, 7), (88, 100), (89, 0)):
        pool.code["v"][int(pool.table[0, t // 32]), 0, t % 32, dim] = math.nan
    check_attn(vr, R, q_len, [n], 1, 4, 32, dtype, window=window, pool=pool, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len,G,H", [([1], [40000], 1, 4), ([8], [9000], 2, 4), ([200], [5000], 1, 4), ([300, 1, 1], [2500, 6000, 70], 2, 8)])
def test_attn_cut(vr, R, dtype, q_len, kv_len, G, H):
    """Keys cut into pieces and joined: several windows of page numbers and scales a wave."""
    check_attn(vr, R, q_len, kv_len, G, H, 64, dtype, seed=kv_len[0])


# ---- attention mass ------------------------------------------------------------------------------

def check_mass(vr, R, q_len, kv_len, G, H, page, dtype, causal=True, window=0, seed=0, pool=None, L=None, inplace=False, kscale=1.0):
    import torch
    say(f"[mass8] q {q_len} kv {kv_len} G={G} H={H} page={page} {dtype} causal={causal} window={window}")
    pool = pool or R.Pool8(kv_len, G, page, seed, kscale=kscale)
    T, S = sum(q_len), len(q_len)
    gen = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((T, H, D), generator=gen).to(R.tdt(dtype))
    lse = R.attn_ref(pool, q, q_len, H, dtype, causal, window)[2].float()
    L = max(kv_len) + 3 if L is None else L
    mass = torch.rand((S, G, L), generator=gen)
    pages, batch = pool.device(vr), pool.batch(vr, q_len)
    md = mass.cuda()
    out = md if inplace else torch.full((S, G, L), 5.0, device="cuda")
    got = vr.paged8_mass(pages, batch, q.cuda(), lse.cuda(), md, causal=causal, window=window, out=None if inplace else out)
    assert got is out
    ref, tol = R.mass_ref(pool, q, q_len, H, lse, mass, dtype, causal, window)
    for s, n in enumerate(kv_len):
        n = min(n, L)
        within(out[s, :, :n], ref[s, :, :n], tol[s, :, :n], f"mass {s}")
        assert torch.equal(out[s, :, n:].cpu(), mass[s, :, n:] if inplace else torch.full((G, L - n), 5.0))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 31, 32, 33, 127, 128, 129, 600])
def test_mass_single_token(vr, R, dtype, n):
    check_mass(vr, R, [1], [n], 2, 8, 32, dtype, seed=n, inplace=n % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,H,page", [(1, 2, 32), (4, 28, 64), (8, 32, 256), (3, 3, 128)])
def test_mass_ragged_batch(vr, R, dtype, G, H, page):
    check_mass(vr, R, [1, 0, 40, 7, 1, 0, 3], [300, 50, 170, 7, 1, 0, 700], G, H, page, dtype, seed=H)
    check_mass(vr, R, [200, 330], [500, 330], G, H, page, dtype, seed=H, inplace=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len,window", [([5, 90], [300, 500], 40), ([300], [700], 1), ([3], [100], 64)])
def test_mass_window_and_all(vr, R, dtype, q_len, kv_len, window):
    check_mass(vr, R, q_len, kv_len, 2, 4, 32, dtype, window=window, seed=window)
    check_mass(vr, R, q_len, kv_len, 2, 4, 32, dtype, causal=False, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mass_edges(vr, R, dtype):
    """Bad pages, rows that see nothing, more sequences than a wave has lanes, lengths beyond the masses."""
    pool = R.Pool8([700, 60], 2, 32, seed=8)
    pool.table[0, 3], pool.table[0, 20] = -1, pool.total
    check_mass(vr, R, [40, 3], [700, 60], 2, 8, 32, dtype, pool=pool, seed=8)
    check_mass(vr, R, [9, 40], [3, 17], 1, 2, 32, dtype, seed=9)
    kv = [1 + (37 * s) % 211 for s in range(150)]
    check_mass(vr, R, [1] * 150, kv, 1, 2, 32, dtype, seed=4)
    check_mass(vr, R, [200], [500], 1, 2, 32, dtype, seed=5, L=333)


# ---- eviction ------------------------------------------------------------------------------------

def check_evict(vr, R, kv_len, keep, G, page, first=0, recent=0, seed=0, mass=None, pool=None, L=None, bad=False):
    import torch
    say(f"[evict8] kv {kv_len} keep={keep} G={G} page={page} first={first} recent={recent}")
    S, need = len(kv_len), (keep + page - 1) // page
    pool = pool or R.Pool8(kv_len, G, page, seed, spare=S * need + 1)
    into = torch.tensor(pool.free[:S * need], dtype=torch.int32).view(S, need)
    if bad:
        pool.table[0, 1], into[0, 0], into[-1, -1] = pool.total, -1, 1 << 30
    L = max(kv_len) + 2 if L is None else L
    if mass is None:
        mass = torch.rand((S, G, L), generator=torch.Generator().manual_seed(seed + 1)) ** 4
    pages = pool.device(vr)
    got = vr.paged8_evict(pages, pool.table.cuda(), torch.tensor(kv_len, dtype=torch.int32).cuda(), mass.cuda(), keep, into.cuda(),
                          first=first, recent=recent)
    want = R.evict_ref(pool, into, mass, keep, first, recent)
    for g, w, name in zip(got, want, ("index", "mass", "length")):
        g = g.cpu()
        assert torch.equal(g.nan_to_num(-7.0), w.nan_to_num(-7.0)) if g.is_floating_point() else torch.equal(g, w), name
    pool.same(pages)


@pytest.mark.parametrize("page", [32, 64, 256])
@pytest.mark.parametrize("keep", [1, 31, 32, 33, 100, 500])
def test_evict(vr, R, page, keep):
    check_evict(vr, R, [300, 40, 1, 0, 33], keep, 2, page, seed=keep)
    check_evict(vr, R, [300, 40, 1, 0, 33], keep, 2, page, first=min(4, keep), recent=min(20, max(0, keep - 4)), seed=keep + 1)


def test_evict_long(vr, R):
    check_evict(vr, R, [9000, 5000], 3000, 3, 128, first=4, recent=32, seed=1)


def test_evict_ties_and_odd_masses(vr, R):
    """Equal masses (zeros of both signs among them) go to the earlier token; negative ones, infinities, NaN last."""
    import torch
    n, G = 5000, 3
    gen = torch.Generator().manual_seed(2)
    mass = torch.randint(0, 4, (2, G, n), generator=gen).float() / 4
    mass[0, 1] = 0.0
    mass[0, 1, ::3] = -0.0
    mass[0, 2, 1::7] = math.nan
    mass[1, 0, 5::11], mass[1, 0, 6::13], mass[1, 0, 7::17] = math.inf, -math.inf, -2.5
    mass[1, 1] = math.nan
    mass[1, 2] = torch.randn(n, generator=gen) * torch.exp2(torch.randint(-140, 120, (n,), generator=gen))
    for keep, first, recent in ((700, 0, 0), (2000, 3, 40), (4999, 1, 1), (5000, 0, 9), (1250, 1250, 0), (64, 4, 60)):
        check_evict(vr, R, [n, n], keep, G, 64, first, recent, seed=keep, mass=mass)


def test_evict_bad_entries(vr, R):
    """Rows of bad pages are zeros, rows for bad pages are dropped; lengths beyond the masses and negative ones are cut."""
    check_evict(vr, R, [300, 300, 70], 100, 2, 32, seed=3, bad=True)
    check_evict(vr, R, [300, 90], 100, 2, 32, seed=4, L=200)
    import torch
    pool = R.Pool8([64, 64], 1, 32, 5, spare=6)
    pool.kv_len = [-5, 64]
    check_evict(vr, R, [-5, 64], 50, 1, 32, seed=5, pool=pool, L=64)


def test_evict_nan_codes(vr, R):
    """NaN rows move as NaN and do not count in their new block's scale."""
    pool = R.Pool8([100], 1, 32, 6, spare=3)
    for t in (3, 40, 77):
        pool.code["k"][int(pool.table[0, t // 32]), 0, t % 32, t] = math.nan
    check_evict(vr, R, [100], 60, 1, 32, seed=6, pool=pool, first=10, recent=50)
