"""GPU parity of the paged cache (norm and rotation, append, attention, gather) against plain
implementations in 64 bits on the host.

Bounds, element by element, with u the rounding of a type (half a step: bf16 2^-8, fp32 2^-24):
  norm and rotation  y: 128 squares are summed in 16 + 3 steps, then root, division and two
                     products: under 16 u32 relative.  Rotation adds two products, a sum and
                     cos, sin right to u32 each: under 4 u32 (|y_i| + |y_j|).  Result rounding u.
  attention          scores: 128 products summed in fp32, 128 u32 c sum|q k|; the exponent's own
                     product and sum 3 u32 (|c x| + |c m|) and the exponential 2 u32.  A weight's
                     error is at most twice that exponent error D (in maximum and in sum).  Weights
                     of bf16 layers are rounded, u, in their products with the values and (few rows)
                     in their sum alike: sum p e (v - o) / sum p, at most u (A + |o|) with A = sum p |v| /
                     sum p (many rows: in the products alone, at most u A).  Sums of n weighted values: n u32.  Together |error| <= u_p (A + |o|) +
                     (4 D + (n + 256) u32) A, and the rounding of the output, u |o|, is of a value
                     that far off: another (1 + u).
  append, gather     copies are exact; a rotated key as above.
"""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

D = 128
U32 = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


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


def tdt(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def theta_of(seed=0):
    import torch
    return (500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float()


def turn64(x, pos, theta):
    import torch
    a = pos.double()[:, None] * theta.double()[None, :]
    c, s = a.cos()[:, None, :], a.sin()[:, None, :]
    return torch.cat([x[..., :64] * c - x[..., 64:] * s, x[..., :64] * s + x[..., 64:] * c], dim=-1)


def pair(x):
    """|x_i| + |x_j| of every rotation pair, at both places."""
    import torch
    y = x.abs()[..., :64] + x.abs()[..., 64:]
    return torch.cat([y, y], dim=-1)


def within(got, ref, tol, what):
    got = got.detach().cpu().double()
    err = (got - ref).abs()
    bad = ~(err <= tol)
    worst = float((err / tol.clamp_min(1e-300)).nan_to_num(0.0).max()) if err.numel() else 0.0
    say(f"  {what}: worst err / bound {worst:.3f}")
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {worst}"


# ---- norm and rotation -----------------------------------------------------------------------

def norm_ref(x, w, pos, theta, eps, dtype):
    """(reference, bound) in 64 bits."""
    y = x.double()
    rel = 0.0
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
        rel = 16 * U32
    tol = rel * y.abs()
    z = y
    if theta is not None:
        z = turn64(y, pos, theta)
        tol = (rel + 4 * U32) * pair(y)
    return z, (tol + U[dtype] * z.abs()) * (1 + U[dtype]) + 1e-38


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,H", [(1, 2), (4, 28), (8, 32), (3, 3)])
@pytest.mark.parametrize("T", [1, 2, 37, 1300])
@pytest.mark.parametrize("norm", ["none", "shared", "each"])
def test_norm_rotate(vr, dtype, G, H, T, norm):
    import torch
    say(f"[norm_rotate] {dtype} G={G} H={H} T={T} {norm}")
    gen = torch.Generator().manual_seed(T * 7 + H)
    x = torch.randn((T, H + 2 * G, D), generator=gen).to(tdt(dtype))
    x[0, 0] = 0                                            # a row of zeros: eps alone
    pos = torch.randint(0, 1 << 20, (T,), generator=gen, dtype=torch.int32)
    theta = theta_of()
    w = [None, None]
    if norm != "none":
        w = [1 + 0.3 * torch.randn((n, D) if norm == "each" else (D,), generator=gen) for n in (H, G)]
    xd = x.cuda()
    cu = lambda t: None if t is None else t.cuda()
    for th in ([theta] if norm == "none" else [theta, None]):
        got = vr.norm_rotate(xd[:, :H], xd[:, H:H + G], pos=pos.cuda(), theta=cu(th), wq=cu(w[0]), wk=cu(w[1]), eps=1e-5)
        for g, src, wt, name in ((got[0], x[:, :H], w[0], "q"), (got[1], x[:, H:H + G], w[1], "k")):
            ref, tol = norm_ref(src, wt, pos, th, 1e-5, dtype)
            within(g, ref, tol, f"{name}{' rotated' if th is not None else ''}")


def test_norm_rotate_far_positions(vr):
    """Angles of positions up to 2^31 - 1, and negative ones, right to fp32."""
    import torch
    pos = torch.tensor([0, 1, -1, (1 << 24) - 1, (1 << 24) + 1, -(1 << 30), (1 << 31) - 1, -(1 << 31)], dtype=torch.int32)
    theta = theta_of()
    theta[3] = 0.0
    x = torch.randn((len(pos), 2, D), generator=torch.Generator().manual_seed(3))
    got, _ = vr.norm_rotate(x.cuda(), pos=pos.cuda(), theta=theta.cuda())
    # the product in 64 bits is itself off by 2^-53 of up to 2^31 radians on either side
    ref, tol = norm_ref(x, None, pos, theta, 0.0, "f32")
    within(got, ref, tol + 2 * 2.0 ** -22 * pair(x.double()), "far")
    near = pos.abs() <= (1 << 24) + 1
    within(got.cpu()[near], ref[near], tol[near] + 2 * 2.0 ** -29 * pair(x.double())[near], "near")


def test_norm_rotate_in_place_and_strided_outputs(vr):
    import torch
    T, G, H = 65, 2, 6
    gen = torch.Generator().manual_seed(5)
    x = torch.randn((T, H + 2 * G, D), generator=gen).bfloat16().cuda()
    pos = torch.arange(T, dtype=torch.int32).cuda()
    theta = theta_of().cuda()
    wq, wk = torch.rand(D, generator=gen).cuda(), torch.rand(D, generator=gen).cuda()
    want = vr.norm_rotate(x[:, :H], x[:, H:H + G], pos=pos, theta=theta, wq=wq, wk=wk)
    out = torch.full((T, H + G + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    vr.norm_rotate(x[:, :H], x[:, H:H + G], pos=pos, theta=theta, wq=wq, wk=wk, q_out=out[:, :H], k_out=out[:, H:H + G])
    assert torch.equal(out[:, :H], want[0]) and torch.equal(out[:, H:H + G], want[1])
    assert (out[:, H + G] == 7).all()
    v = x[:, H + G:].clone()
    vr.norm_rotate(x[:, :H], x[:, H:H + G], pos=pos, theta=theta, wq=wq, wk=wk, q_out=x[:, :H], k_out=x[:, H:H + G])
    assert torch.equal(x[:, :H], want[0]) and torch.equal(x[:, H:H + G], want[1]) and torch.equal(x[:, H + G:], v)
    # one side alone, and a broadcast row (stride 0)
    only_q = vr.norm_rotate(want[0], pos=pos, theta=theta)
    assert only_q[1] is None
    only_k = vr.norm_rotate(None, want[1], pos=pos, theta=theta)
    both = vr.norm_rotate(want[0], want[1], pos=pos, theta=theta)
    assert torch.equal(only_q[0], both[0]) and torch.equal(only_k[1], both[1])
    row = want[0][:1].expand(T, H, D)
    assert torch.equal(vr.norm_rotate(row, pos=pos, theta=theta)[0], vr.norm_rotate(row.contiguous(), pos=pos, theta=theta)[0])


# ---- a pool, its sequences, and the references over them ----------------------------------------

class Pool:
    """Host copies of pages in shuffled order; slots that no sequence uses hold `junk`."""

    def __init__(self, kv_len, G, page, dtype, seed=0, junk=float("nan"), width=None, scale=1.0):
        import torch
        gen = torch.Generator().manual_seed(seed)
        need = [(n + page - 1) // page for n in kv_len]
        total = sum(need) + 2
        self.k = torch.full((total, G, page, D), junk, dtype=tdt(dtype))
        self.v = torch.full((total, G, page, D), junk, dtype=tdt(dtype))
        width = max(need + [1]) if width is None else width
        self.table = torch.full((len(kv_len), width), -1, dtype=torch.int32)
        order = torch.randperm(total, generator=gen)
        at = 0
        for s, (n, m) in enumerate(zip(kv_len, need)):
            self.table[s, :m] = order[at:at + m].int()
            at += m
            for t0 in range(0, n, page):
                c = min(page, n - t0)
                p = int(self.table[s, t0 // page])
                self.k[p, :, :c] = (scale * torch.randn((G, c, D), generator=gen)).to(self.k.dtype)
                self.v[p, :, :c] = torch.randn((G, c, D), generator=gen).to(self.v.dtype)
        self.kv_len, self.G, self.page, self.dtype = list(kv_len), G, page, dtype

    def rows(self, s, n=None):
        """(K, V) [n][G][d] of sequence s; a bad page's rows are None-marked by `ok` [n]."""
        import torch
        n = self.kv_len[s] if n is None else n
        t = torch.arange(n)
        pg = self.table[s][t // self.page].long()
        ok = (pg >= 0) & (pg < self.k.shape[0])
        pg = torch.where(ok, pg, 0)
        return self.k[pg, :, t % self.page], self.v[pg, :, t % self.page], ok

    def device(self, vr, q_len, pad=0):
        import torch
        start = torch.tensor([pad + sum(q_len[:s]) for s in range(len(q_len) + 1)], dtype=torch.int32)
        pages = vr.PagedCache(self.k.cuda(), self.v.cuda())
        batch = vr.PagedBatch(self.table.cuda(), torch.tensor(self.kv_len, dtype=torch.int32).cuda(), start.cuda())
        return pages, batch


def attn_ref(pool, q, q_len, H, causal=True, window=0, scale=None):
    """(reference, bound) of every new token, 64 bits, keys that a token does not see left out."""
    import torch
    G = pool.G
    c = 1 / math.sqrt(D) if scale is None else scale
    T = sum(q_len)
    ref = torch.zeros((T, H, D), dtype=torch.float64)
    tol = torch.zeros((T, H, D), dtype=torch.float64)
    at = 0
    for s, m in enumerate(q_len):
        n = pool.kv_len[s]
        K, V, ok = pool.rows(s)
        for i in range(m):
            p = n - m + i
            t = torch.arange(n)
            see = ok.clone()
            if causal:
                see &= t <= p
                if window:
                    see &= p - t < window
            t = t[see]
            if not len(t):
                continue
            for h in range(H):
                k, v = K[t, h // (H // G)].double(), V[t, h // (H // G)].double()
                x = q[at + i, h].double()
                sc = (k @ x) * c
                w = torch.softmax(sc, 0)
                o = w @ v
                A = w @ v.abs()
                mag = c * (k.abs() @ x.abs())
                dx = float((128 * U32 * mag + 3 * U32 * (sc.abs() + sc.abs().max())).max()) + 2 * U32
                u = U[pool.dtype]
                e = (u if pool.dtype == "bf16" else 0) * (A + o.abs()) + (4 * dx + (len(t) + 256) * U32) * A
                ref[at + i, h] = o
                tol[at + i, h] = (e + u * o.abs()) * (1 + u) + 1e-38
        at += m
    return ref, tol


def check_attn(vr, q_len, kv_len, G, H, page, dtype, causal=True, window=0, seed=0, pool=None, scale=None, qscale=2.0):
    import torch
    say(f"[attn] q {q_len} kv {kv_len} G={G} H={H} page={page} {dtype} causal={causal} window={window}")
    pool = pool or Pool(kv_len, G, page, dtype, seed)
    q = (qscale * torch.randn((sum(q_len), H, D), generator=torch.Generator().manual_seed(seed + 1))).to(tdt(dtype))
    pages, batch = pool.device(vr, q_len)
    out = vr.paged_attn(pages, batch, q.cuda(), causal=causal, window=window, scale=scale)
    torch.cuda.synchronize()
    ref, tol = attn_ref(pool, q, q_len, H, causal, window, scale)
    within(out, ref, tol, "out")
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 511, 513, 2100])
def test_attn_single_token(vr, dtype, n):
    check_attn(vr, [1], [n], 2, 8, 16, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 16, 31, 33, 64, 65, 100, 130, 257])
def test_attn_prompt(vr, dtype, n):
    check_attn(vr, [n], [n], 1, 3, 32, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,H,page", [(1, 2, 16), (4, 28, 64), (8, 32, 256), (3, 3, 128), (1, 40, 32)])
def test_attn_ragged_batch(vr, dtype, G, H, page):
    """Chunks, prompts, single tokens and sequences with nothing new or nothing at all, together."""
    check_attn(vr, [1, 0, 40, 7, 1, 0, 3], [300, 50, 170, 7, 1, 0, 1000], G, H, page, dtype, seed=H)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([1, 1, 2], [1500, 40, 700]), ([60], [1700]), ([130, 5], [900, 1100])])
@pytest.mark.parametrize("window", [1, 16, 63, 64, 65, 500])
def test_attn_window(vr, dtype, q_len, kv_len, window):
    check_attn(vr, q_len, kv_len, 2, 4, 16, dtype, window=window, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([1], [700]), ([5, 2], [33, 2000]), ([70], [300]), ([150], [40])])
def test_attn_all_keys(vr, dtype, q_len, kv_len):
    check_attn(vr, q_len, kv_len, 2, 6, 32, dtype, causal=False, seed=kv_len[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([3, 9], [1, 0]), ([40, 2], [17, 1])])
def test_attn_rows_that_see_nothing(vr, dtype, q_len, kv_len):
    """More new tokens than the cache holds: the first ones stand before it and get zeros."""
    out = check_attn(vr, q_len, kv_len, 2, 4, 16, dtype, seed=9)
    assert (out[:q_len[0] - kv_len[0]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_many_sequences(vr, dtype):
    """More than 64 sequences (the lengths are scanned 64 at a time), unlike lengths."""
    kv = [1 + (37 * s) % 211 for s in range(150)]
    check_attn(vr, [1] * 150, kv, 1, 2, 16, dtype, seed=4)
    check_attn(vr, [min(k, 1 + s % 50) for s, k in enumerate(kv)], kv, 1, 2, 16, dtype, seed=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [[1, 1], [90, 30]])
def test_attn_large_scores(vr, dtype, q_len):
    """Logits in the hundreds, of both signs: the maximum moves late and by far."""
    pool = Pool([900, 333], 2, 64, dtype, seed=6)
    p, at = int(pool.table[0, 13]), 850 % 64
    pool.k[p, :, at] *= 8
    check_attn(vr, q_len, [900, 333], 2, 8, 64, dtype, pool=pool, seed=6, qscale=20.0)
    check_attn(vr, q_len, [900, 333], 2, 8, 64, dtype, pool=pool, seed=6, scale=1e-3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [[1, 4], [60, 45]])
def test_attn_bad_pages(vr, dtype, q_len):
    """Entries that name no page: their tokens are left out (a sequence of bad pages alone: zeros)."""
    pool = Pool([700, 500], 2, 32, dtype, seed=8)
    big = pool.k.shape[0]
    for i, bad in ((0, -1), (3, big), (4, -(1 << 31)), (9, (1 << 31) - 1), (21, big + 7)):
        pool.table[0, i] = bad
    check_attn(vr, q_len, [700, 500], 2, 8, 32, dtype, pool=pool, seed=8)
    pool.table[1] = -1
    out = check_attn(vr, q_len, [700, 500], 2, 8, 32, dtype, pool=pool, seed=8)
    assert (out[q_len[0]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,window", [([50], 0), ([3], 0), ([50], 20), ([3], 20)])
@pytest.mark.parametrize("odd", [float("inf"), float("-inf"), float("nan")])
def test_attn_odd_values_in_unseen_places(vr, dtype, q_len, window, odd):
    """Infinities and NaN in keys and values of later tokens, of tokens behind the window and of
    slots behind the end reach no row that does not see them."""
    import torch
    n = 333
    pool = Pool([n], 2, 16, dtype, seed=11, junk=odd)
    m = q_len[0]
    later = n - m + m // 2                                 # seen by the second half of the new tokens alone
    def slot(t):
        return int(pool.table[0, t // 16]), t % 16
    spoiled = [later] + ([n - m - 30] if window else [])   # that one lies behind every row's window
    keep = {t: (pool.k[slot(t)[0], :, slot(t)[1]].clone(), pool.v[slot(t)[0], :, slot(t)[1]].clone()) for t in spoiled}
    q = torch.randn((m, 4, D), generator=torch.Generator().manual_seed(12)).to(tdt(dtype))
    ref, tol = attn_ref(pool, q, q_len, 4, True, window)
    for t in spoiled:
        p, i = slot(t)
        pool.k[p, 0, i, 5] = odd
        pool.v[p, 1, i, 7] = odd
        pool.v[p, 0, i] = odd
    pages, batch = pool.device(vr, q_len)
    out = vr.paged_attn(pages, batch, q.cuda(), window=window)
    half = m // 2
    within(out[:half], ref[:half], tol[:half], f"rows before the odd token ({odd})")
    if window:
        for t in spoiled[:1]:
            p, i = slot(t)
            pool.k[p, :, i], pool.v[p, :, i] = keep[t]
        pages, batch = pool.device(vr, q_len)
        within(vr.paged_attn(pages, batch, q.cuda(), window=window), ref, tol, "behind the window")
    else:
        assert not torch.isfinite(out[half:, :, 7].float()).all()       # who sees it, has it


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [[1, 2], [70, 33]])
def test_attn_padding_strides_and_streams(vr, dtype, q_len):
    """Padded rows before and behind the sequences are left as they were; strided queries, outputs
    and table rows; a stream of its own."""
    import torch
    H, G, pad = 6, 2, 3
    kv = [400, 95]
    pool = Pool(kv, G, 32, dtype, seed=13)
    m = sum(q_len)
    T = pad + m + 5
    fused = torch.randn((T, H + 2 * G, D), generator=torch.Generator().manual_seed(2)).to(tdt(dtype))
    wide = torch.full((2, pool.table.shape[1] + 3), 77777, dtype=torch.int32)
    wide[:, :pool.table.shape[1]] = pool.table
    pages, batch = pool.device(vr, q_len, pad=pad)
    table = wide.cuda()[:, :pool.table.shape[1]]
    batch = vr.PagedBatch(table, batch.kv_len, batch.q_start)
    out = torch.full((T, H + 1, D), 5.0, dtype=tdt(dtype), device="cuda")
    fd = fused.cuda()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        vr.paged_attn(pages, batch, fd[:, :H], out=out[:, :H])
    st.synchronize()
    ref, tol = attn_ref(pool, fused[pad:pad + m, :H], q_len, H)
    within(out[pad:pad + m, :H], ref, tol, "strided")
    assert (out[:pad] == 5).all() and (out[pad + m:] == 5).all() and (out[:, H] == 5).all()


def test_attn_same_bits_again(vr):
    """No result depends on the order in which workgroups run."""
    import torch
    for q_len, kv in (([1] * 3, [4000, 1, 700]), ([100, 1], [3000, 2000])):
        for dtype in ("bf16", "f32"):
            pool = Pool(kv + [0] * (len(q_len) - len(kv)), 2, 64, dtype, seed=3)
            q = torch.randn((sum(q_len), 8, D), generator=torch.Generator().manual_seed(1)).to(tdt(dtype)).cuda()
            pages, batch = pool.device(vr, q_len)
            a = vr.paged_attn(pages, batch, q)
            assert all(torch.equal(a, vr.paged_attn(pages, batch, q)) for _ in range(3))


# ---- append and gather -------------------------------------------------------------------------

def append_ref(pool, k, v, q_len, kv_len, theta):
    """(pools after, bound on the keys) with rows that have no slot dropped."""
    import torch
    K, V = pool.k.double().clone(), pool.v.clone()
    tol = torch.zeros_like(K)
    at = 0
    for s, m in enumerate(q_len):
        for i in range(m):
            t = kv_len[s] - m + i
            if 0 <= t and kv_len[s] <= pool.table.shape[1] * pool.page:
                p = int(pool.table[s, t // pool.page])
                if 0 <= p < K.shape[0]:
                    row = k[at + i].double()
                    b = torch.zeros_like(row)
                    if theta is not None:
                        z = turn64(row[None], torch.tensor([t]), theta)[0]
                        b = (4 * U32 * pair(row) + U[pool.dtype] * z.abs()) * (1 + U[pool.dtype])
                        row = z
                    K[p, :, t % pool.page], tol[p, :, t % pool.page] = row, b
                    V[p, :, t % pool.page] = v[at + i]
        at += m
    return K, V, tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,page", [(1, 16), (8, 64), (3, 256)])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("q_len,kv_len", [([1], [1]), ([1, 1, 1], [40, 1, 17]), ([30, 0, 5, 2], [30, 9, 300, 1]),
                                          ([700], [1900])])
def test_append(vr, dtype, G, page, rotate, q_len, kv_len):
    import torch
    say(f"[append] {dtype} G={G} page={page} rotate={rotate} q {q_len} kv {kv_len}")
    gen = torch.Generator().manual_seed(G + page)
    pool = Pool(kv_len, G, page, dtype, seed=1, junk=3.0)
    if len(kv_len) > 1 and page == 16:
        pool.table[0, -1] = pool.k.shape[0]                # a page past the pool: its rows are dropped
        if kv_len[0] > 16:
            pool.table[0, 0] = -5
    pad = 2
    x = torch.randn((pad + sum(q_len) + 3, 2 * G + 1, D), generator=gen).to(tdt(dtype))
    theta = theta_of() if rotate else None
    pages, batch = pool.device(vr, q_len, pad=pad)
    xd = x.cuda()
    vr.paged_append(pages, batch, xd[:, :G], xd[:, G:2 * G], theta=None if theta is None else theta.cuda())
    K, V, tol = append_ref(pool, x[pad:, :G], x[pad:, G:2 * G], q_len, kv_len, theta)
    assert torch.equal(pages.v.cpu(), V)
    if rotate:
        within(pages.k, K, tol, "keys")
    else:
        assert torch.equal(pages.k.cpu().double(), K)


def test_append_lengths_outside_the_table(vr):
    """A length past the table, or below zero: nothing is written for that sequence; rows whose
    position would be negative are dropped."""
    import torch
    pool = Pool([64, 64, 64], 2, 16, "bf16", seed=2, junk=1.0)
    x = torch.randn((12, 2, D), generator=torch.Generator().manual_seed(3)).bfloat16()
    for lens in ([65, 64, 2], [1 << 30, -4, 0], [(1 << 31) - 1, -(1 << 31), 64]):
        pages, batch = pool.device(vr, [4, 4, 4])
        batch.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        vr.paged_append(pages, batch, x.cuda(), x.cuda())
        K, V, _ = append_ref(pool, x, x, [4, 4, 4], lens, None)
        assert torch.equal(pages.k.cpu().double(), K) and torch.equal(pages.v.cpu(), V), lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,page,n", [(1, 16, 1), (2, 16, 33), (8, 64, 1000), (4, 256, 256), (3, 32, 0)])
def test_gather(vr, dtype, G, page, n):
    import torch
    pool = Pool([n], G, page, dtype, seed=n)
    pages, batch = pool.device(vr, [0])
    K, V = vr.paged_gather(pages, batch.table[0], n)
    k, v, _ = pool.rows(0)
    assert K.shape == (n, G, D) and torch.equal(K.cpu(), k) and torch.equal(V.cpu(), v)
    if n > page:
        pool.table[0, 1], pool.table[0, 0] = -1, pool.k.shape[0]
        pages, batch = pool.device(vr, [0])
        K, V = vr.paged_gather(pages, batch.table[0], n)
        k, v, ok = pool.rows(0)
        k[~ok], v[~ok] = 0, 0
        assert torch.equal(K.cpu(), k) and torch.equal(V.cpu(), v)


# ---- together, as they are used ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_in_chunks_then_compressed(vr, dtype):
    """A prompt arrives in chunks beside a second sequence that decodes: norm and rotate, append,
    attend; then the prompt is gathered and compressed, and decode over the codec at full budget
    agrees with attention over the pages."""
    import torch
    G, H, page, n, w = 2, 8, 32, 700, 32
    gen = torch.Generator().manual_seed(21)
    dt = tdt(dtype)
    theta = theta_of()
    wq, wk = 1 + 0.1 * torch.randn(D, generator=gen), 1 + 0.1 * torch.randn(D, generator=gen)
    x = torch.randn((n, H + 2 * G, D), generator=gen).to(dt)         # the prompt's projections
    y = torch.randn((40, H + 2 * G, D), generator=gen).to(dt)        # the other sequence's
    pages = vr.new_pages(40, G, page, dtype)
    table = torch.randperm(40, generator=gen).int()[:2 * 23].reshape(-1)[:40]
    tab = torch.stack([table[:23], torch.cat([table[23:25], torch.full((21,), -1)])]).int().cuda()
    done, other, outs, ys = 0, 0, [], []
    qw = None
    for m in (256, 300, 1, 143):
        rows = torch.cat([x[done:done + m], y[other:other + 1]]).cuda()
        done, other = done + m, other + 1
        batch = vr.PagedBatch(tab, torch.tensor([done, other], dtype=torch.int32).cuda(),
                              torch.tensor([0, m, m + 1], dtype=torch.int32).cuda())
        pos = torch.cat([torch.arange(done - m, done), torch.tensor([other - 1])]).int().cuda()
        q, k = vr.norm_rotate(rows[:, :H], rows[:, H:H + G], pos=pos, theta=theta.cuda(), wq=wq.cuda(), wk=wk.cuda())
        vr.paged_append(pages, batch, k, rows[:, H + G:])
        o = vr.paged_attn(pages, batch, q)
        outs.append(o[:m])
        ys.append(o[m:])
        qw = q[:m] if qw is None else torch.cat([qw, q[:m]])
    assert done == n
    # the same from what the operators were documented to do, in 64 bits on their own stored rows
    zk, _ = norm_ref(x[:, H:H + G], wk, torch.arange(n), theta, 1e-6, dtype)
    K, V = vr.paged_gather(pages, tab[0], n)
    zk, tk = norm_ref(x[:, H:H + G], wk, torch.arange(n), theta, 1e-6, dtype)
    within(K, zk, tk, "keys in the pages")
    assert torch.equal(V.cpu(), x[:, H + G:])
    pool = Pool([n, other], G, page, dtype)
    pool.k, pool.v, pool.table = pages.k.cpu(), pages.v.cpu(), tab.cpu()
    ref, tol = attn_ref(pool, torch.cat([qw.cpu(), torch.zeros((other, H, D), dtype=dt)]), [n, other], H)
    within(torch.cat(outs), ref[:n], tol[:n], "prompt")
    # handed to the codec at full budget (every token at full rank): decode is the same attention
    shape = vr.Shape(n=n, G=G, H=H, w=w, r_min=16, kappa_pct=100, dtype=dtype,
                     rope_theta=tuple(float(t) for t in theta))
    P = torch.linalg.qr(torch.randn((2, G, D, D), generator=gen))[0].contiguous().cuda()
    cache = vr.compress(shape, K, V, qw[n - w:].contiguous(), P[0].contiguous(), P[1].contiguous())
    q = torch.randn((1, H, D), generator=gen).to(dt).cuda()
    a = vr.decode(shape, [cache], q, P[0].contiguous(), P[1].contiguous())
    batch = vr.PagedBatch(tab[:1], torch.tensor([n], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda())
    b = vr.paged_attn(pages, batch, q, causal=False)
    e = float((a.double() - b.double()).abs().amax() / b.double().abs().amax())
    say(f"  decode over the codec against the pages: {e:.2e}")
    assert e <= (2e-2 if dtype == "bf16" else 1e-4)        # the rotary codec's own parity bars


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps_follow_new_lengths(vr, dtype):
    """A decode step (norm and rotation, append, attention) captured once, its lengths, positions and
    inputs renewed between replays; two graphs over one pool; eager work in between."""
    import torch
    G, H, page, S, pad = 2, 8, 16, 3, 1
    dt = tdt(dtype)
    gen = torch.Generator().manual_seed(31)
    theta = theta_of().cuda()
    lens = [30, 1, 700]
    pool = Pool([v + 20 for v in lens], G, page, dtype, seed=7, junk=0.0)
    pages, _ = pool.device(vr, [1] * S)
    eager = vr.PagedCache(pages.k.clone(), pages.v.clone())
    x = torch.zeros((S + pad, H + 2 * G, D), dtype=dt, device="cuda")
    kv = torch.tensor(lens, dtype=torch.int32).cuda()
    pos = torch.zeros(S + pad, dtype=torch.int32, device="cuda")
    batch = vr.PagedBatch(pool.table.cuda(), kv, torch.arange(S + 1, dtype=torch.int32).cuda())
    out = torch.zeros((S + pad, H, D), dtype=dt, device="cuda")

    def step(pg, o):
        q, k = vr.norm_rotate(x[:, :H], x[:, H:H + G], pos=pos, theta=theta)
        vr.paged_append(pg, batch, k, x[:, H + G:])
        vr.paged_attn(pg, batch, q, out=o)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(pages, out)
    side.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(pages, out)
        graphs.append(g)
    pages.k.copy_(eager.k)
    pages.v.copy_(eager.v)
    for i in range(6):
        now = [v + i + 1 for v in lens]
        kv.copy_(torch.tensor(now, dtype=torch.int32))
        pos[:S] = kv - 1
        x.copy_(torch.randn(x.shape, generator=gen).to(dt))
        graphs[i % 2].replay()
        got = out.clone()
        want = torch.zeros_like(out)
        step(eager, want)
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
        assert torch.equal(pages.k, eager.k) and torch.equal(pages.v, eager.v), i


def test_two_streams_at_once(vr):
    """Two calls in flight on two streams, each with workspaces of its own."""
    import torch
    pool = Pool([5000, 4000], 2, 64, "bf16", seed=17)
    pages, batch = pool.device(vr, [1, 1])
    qs = [torch.randn((2, 8, D), generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in range(2)]
    want = [vr.paged_attn(pages, batch, q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(8):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(vr.paged_attn(pages, batch, qs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])


# ---- the far ends of the ranges, and what the binding refuses --------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 5, 8, 70])
def test_attn_seen_infinities(vr, dtype, m):
    """Infinite values reach the rows that see them, in their own dims and heads, and nothing else: rows of
    one token, of up to 16, of up to 32 and many."""
    import torch
    n, G, H = 333, 2, 8
    pool = Pool([n], G, 16, dtype, seed=41)
    q = torch.randn((m, H, D), generator=torch.Generator().manual_seed(42)).to(tdt(dtype))
    ref, tol = attn_ref(pool, q, [m], H)
    t = n - m + m // 2
    p, i = int(pool.table[0, t // 16]), t % 16
    up, down = [0, 7, 33, 64, 100, 127], [1, 18, 31, 47, 95, 126]
    pool.v[p, 1, i, up] = float("inf")
    pool.v[p, 1, i, down] = float("-inf")
    pages, batch = pool.device(vr, [m])
    out = vr.paged_attn(pages, batch, q.cuda()).cpu().double()
    hit = torch.zeros((m, H, D), dtype=torch.bool)
    hit[m // 2:, 4:, up + down] = True
    assert (out[m // 2:, 4:][..., up] == float("inf")).all() and (out[m // 2:, 4:][..., down] == float("-inf")).all()
    within(out[~hit], ref[~hit], tol[~hit], "the others")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_many_sequences_some_cut(vr, dtype):
    """150 sequences with long ones and chunks among the first and the last 64."""
    kv = [1 + (37 * s) % 211 for s in range(150)]
    q = [1] * 150
    for s, (m, n) in {2: (1, 3000), 5: (90, 700), 63: (1, 1200), 64: (3, 900), 100: (70, 70), 127: (0, 50), 149: (1, 2500)}.items():
        q[s], kv[s] = m, n
    check_attn(vr, q, kv, 1, 4, 16, dtype, seed=19)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_many_heads(vr, dtype):
    """One KV head with more query heads than a tile has rows; scales at the lower end."""
    check_attn(vr, [1, 2], [300, 50], 1, 300, 16, dtype, seed=23)
    check_attn(vr, [1, 20], [300, 50], 1, 4, 16, dtype, seed=24, scale=2.0 ** -100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(vr, dtype):
    """Pools of more than 2^32 bytes and 2^31 elements: the last pages give what the first give."""
    import torch
    G, H, page = 8, 32, 64
    n_pages = (1 << 31) // (G * page * D) + 40
    lens, q_len = [500, 90, 700], [1, 90, 33]
    pool = Pool(lens, G, page, dtype, seed=29)
    small, batch = pool.device(vr, q_len)
    far = vr.PagedCache(*(torch.empty((n_pages, G, page, D), dtype=tdt(dtype), device="cuda") for _ in range(2)))
    assert far.k.numel() > 1 << 31 and far.k.numel() * far.k.element_size() > 1 << 32
    shift = n_pages - pool.k.shape[0]
    far.k[shift:], far.v[shift:] = small.k, small.v
    ftab = torch.where(pool.table >= 0, pool.table + shift, pool.table).cuda()
    fbatch = vr.PagedBatch(ftab, batch.kv_len, batch.q_start)
    gen = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((sum(q_len), h, D), generator=gen).to(tdt(dtype)).cuda() for h in (H, G, G))
    theta = theta_of().cuda()
    vr.paged_append(small, batch, k, v, theta)
    vr.paged_append(far, fbatch, k, v, theta)
    same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))      # unused slots hold NaN
    assert same(far.k[shift:], small.k) and same(far.v[shift:], small.v)
    assert torch.equal(vr.paged_attn(far, fbatch, q), vr.paged_attn(small, batch, q))
    for s, n in enumerate(lens):
        a, b = vr.paged_gather(far, ftab[s], n), vr.paged_gather(small, batch.table[s], n)
        assert same(a[0], b[0]) and same(a[1], b[1])


def test_norm_rotate_more_blocks_than_the_grid(vr):
    """2^24 + 5 rows of one head: the workgroups go round, and the last rows are right."""
    import torch
    T = (1 << 24) + 5
    x = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    theta = theta_of().cuda()
    gen = torch.Generator().manual_seed(3)
    parts = [slice(0, 40), slice((1 << 24) - 20, T), slice(1 << 23, (1 << 23) + 30)]
    for s in parts:
        x[s] = torch.randn((s.stop - s.start, 1, D), generator=gen).bfloat16().cuda()
        pos[s] = torch.randint(0, 1 << 20, (s.stop - s.start,), generator=gen, dtype=torch.int32).cuda()
    out = vr.norm_rotate(x, pos=pos, theta=theta)[0]
    for s in parts:
        ref, tol = norm_ref(x[s].cpu(), None, pos[s].cpu(), theta.cpu(), 0, "bf16")
        within(out[s], ref, tol, str(s))


def test_binding_refuses(vr):
    """Wrong types, shapes, strides and devices raise before anything is enqueued; nothing is written."""
    import torch
    G, H, page, T = 2, 4, 16, 3
    pages = vr.new_pages(4, G, page)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    batch = vr.PagedBatch(i32(0, 1).view(1, 2), i32(20), i32(0, T))
    q, k, v = (torch.ones((T, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, G, G))
    th, pos = theta_of().cuda(), i32(0, 1, 2)
    wide = torch.ones((T, H, 2 * D), dtype=torch.bfloat16, device="cuda")
    bad = [
        lambda: vr.PagedCache(pages.k, pages.v[:2]), lambda: vr.PagedCache(pages.k, pages.v.float()),
        lambda: vr.PagedCache(pages.k.half(), pages.v.half()), lambda: vr.PagedCache(pages.k.transpose(1, 2), pages.v.transpose(1, 2)),
        lambda: vr.PagedCache(pages.k.cpu(), pages.v.cpu()), lambda: vr.new_pages(4, G, 24) and vr.paged_gather(vr.new_pages(4, G, 24), i32(0), 1),
        lambda: vr.PagedBatch(i32(0, 1), i32(20), i32(0, 3)), lambda: vr.PagedBatch(i32(0, 1).view(1, 2).long(), i32(20), i32(0, 3)),
        lambda: vr.PagedBatch(i32(0, 1).view(1, 2), i32(20, 20), i32(0, 3)), lambda: vr.PagedBatch(i32(0, 1).view(1, 2), i32(20), i32(0)),
        lambda: vr.PagedBatch(i32(0, 1).view(1, 2), i32(20).cpu(), i32(0, 3)),
        lambda: vr.PagedBatch(i32(0, 1, 2, 3).view(1, 4)[:, ::2], i32(20), i32(0, 3)),
        lambda: vr.norm_rotate(None), lambda: vr.norm_rotate(q, theta=th), lambda: vr.norm_rotate(q, pos=pos.long(), theta=th),
        lambda: vr.norm_rotate(q, pos=pos[:2], theta=th), lambda: vr.norm_rotate(q, pos=pos, theta=th[:32]),
        lambda: vr.norm_rotate(q, pos=pos, theta=th.double()), lambda: vr.norm_rotate(q.half()), lambda: vr.norm_rotate(q, k.float()),
        lambda: vr.norm_rotate(q, k[:2]), lambda: vr.norm_rotate(q, wq=th), lambda: vr.norm_rotate(q, wk=torch.ones(D, device="cuda")),
        lambda: vr.norm_rotate(q, wq=torch.ones((G, D), device="cuda")), lambda: vr.norm_rotate(wide[..., ::2]),
        lambda: vr.norm_rotate(q, q_out=k), lambda: vr.norm_rotate(q, q_out=q.float()), lambda: vr.norm_rotate(q, eps=-1.0),
        lambda: vr.norm_rotate(q[..., :64]), lambda: vr.norm_rotate(wide.view(-1)[4:4 + T * H * D].view(T, H, D)),
        lambda: vr.paged_append(pages, batch, k.float(), v), lambda: vr.paged_append(pages, batch, k, v[:2]),
        lambda: vr.paged_append(pages, batch, q, v), lambda: vr.paged_append(pages, batch, k.cpu(), v),
        lambda: vr.paged_append(pages, batch, k, v, theta=th[1:33]), lambda: vr.paged_attn(pages, batch, q.float()),
        lambda: vr.paged_attn(pages, batch, q[0]), lambda: vr.paged_attn(pages, batch, q[:, :3]), lambda: vr.paged_attn(pages, batch, q, out=k),
        lambda: vr.paged_attn(pages, batch, q, out=q), lambda: vr.paged_attn(pages, batch, q, window=-1),
        lambda: vr.paged_attn(pages, batch, q, causal=False, window=4), lambda: vr.paged_attn(pages, batch, q, scale=0.0),
        lambda: vr.paged_attn(pages, batch, q, scale=float("nan")), lambda: vr.paged_attn(pages, batch, q, out=q.cpu()),
        lambda: vr.paged_attn(pages, vr.PagedBatch(i32(*range(40)).view(1, 40), i32(20), i32(0, T)), q,
                              workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
        lambda: vr.paged_gather(pages, i32(0, 1), -1), lambda: vr.paged_gather(pages, i32(0, 1), 33),
        lambda: vr.paged_gather(pages, i32(0, 1).view(1, 2), 3), lambda: vr.paged_gather(pages, i32(0, 1).cpu(), 3),
        lambda: vr.paged_gather(pages, i32(0, 1), 3, K=k[:2]), lambda: vr.paged_gather(pages, i32(0, 1), 3, V=v.float()),
        lambda: vr.paged_gather(pages, i32(0, 1), 3, K=wide[:, :G, ::2]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(vr.VarRateError):
            call()
            say(f"call {i} was not refused")
    torch.cuda.synchronize()
    assert (pages.k == 0).all() and (pages.v == 0).all() and (q == 1).all() and (k == 1).all()


def test_tensors_of_a_handle_stay(vr):
    """A handle keeps the tensors whose addresses its calls use: they cannot be replaced, and live as long as it does."""
    import torch
    pages = vr.new_pages(3, 1, 16)
    batch = vr.PagedBatch(torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"),
                          torch.tensor([0, 1], dtype=torch.int32).cuda())
    for handle, names in ((pages, ("k", "v")), (batch, ("table", "kv_len", "q_start"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(handle, name, getattr(handle, name).clone())
    x = torch.randn((1, 1, D), device="cuda").bfloat16()
    vr.paged_append(pages, batch, x, x)
    assert torch.equal(vr.paged_attn(pages, batch, x), x)              # one key: its value


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_thousands_of_sequences(vr, dtype):
    """3000 sequences, most of them short, one long and one with a chunk of new tokens."""
    import torch
    S = 3000
    kv = [1 + (7 * s) % 23 for s in range(S)]
    q_len = [1] * S
    q_len[1500], kv[1500] = 40, 900
    kv[2900] = 1300
    pool = Pool(kv, 1, 16, dtype, seed=51)
    q = torch.randn((sum(q_len), 4, D), generator=torch.Generator().manual_seed(52)).to(tdt(dtype))
    pages, batch = pool.device(vr, q_len)
    out = vr.paged_attn(pages, batch, q.cuda()).cpu()
    at = 0
    for s in range(S):
        if s % 97 == 0 or s in (1499, 1500, 1501, 2900, 2999):
            one = Pool.__new__(Pool)
            one.__dict__.update(pool.__dict__)
            one.table, one.kv_len = pool.table[s:s + 1], [kv[s]]
            ref, tol = attn_ref(one, q[at:at + q_len[s]], [q_len[s]], 4)
            within(out[at:at + q_len[s]], ref, tol, f"sequence {s}")
        at += q_len[s]
