"""GPU tests of the paged cache at the edges of its ranges: scores of any size.  References, bounds and pools are those of
test_gpu_paged.py."""
import math

import pytest

from test_gpu_paged import D, U, U32, Pool, attn_ref, say, tdt, vr, within  # noqa: F401

pytestmark = pytest.mark.gpu

# (new tokens, cached tokens, table entries or None for as many as are needed) by the form that serves them: few rows
# and many, in tables too short to cut (8 pages of 32) and in long ones
FORMS = {"few": ([1], [200], 8), "few cut": ([2], [6000], None), "many": ([70], [200], 8), "many cut": ([70], [6000], None)}


def one_call(vr, pool, q, q_len, **kw):
    import torch
    pages, batch = pool.device(vr, q_len)
    out = vr.paged_attn(pages, batch, q.cuda(), **kw)
    torch.cuda.synchronize()
    return out.cpu().double()


def mean_of(pool, m, which=None):
    """(the plain mean of the values that each of the last m tokens sees, and a bound on it): weights are alike, so that
    only they (bf16, in their products: u A), the sums (n roundings of 32 bits at most) and the output round.
    which: of those keys alone."""
    import torch
    _, V, _ = pool.rows(0)
    n = len(V)
    keep = torch.ones(n, dtype=torch.bool) if which is None else which
    ref, tol = [], []
    for i in range(n - m + 1, n + 1):
        v = V[:i][keep[:i]].double()[:, 0]
        ref.append(v.mean(0))
        tol.append(((n + 256) * U32 + (U["bf16"] if pool.dtype == "bf16" else 0)) * v.abs().mean(0))
    ref, tol = torch.stack(ref)[:, None], torch.stack(tol)[:, None]
    u = U[pool.dtype]
    return ref, (tol + u * ref.abs()) * (1 + u) + 1e-38


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", [-20, 20, 27, 28, 30, 40, 93, 100])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_attn_equal_scores_of_any_size(vr, dtype, form, power, sign):
    """scale <q, k> of about 2^(35 + power) for every key, <q, k> itself (1.4 x 2^35) within fp32: whichever form and cut
    serves the call, the mean of the values."""
    import torch
    q_len, kv_len, width = FORMS[form]
    say(f"[scores] {dtype} {form} 2^{power} {sign}")
    pool = Pool(kv_len, 1, 32, dtype, seed=3, width=width)
    pool.k[:] = torch.where(pool.k.isnan(), pool.k, torch.full_like(pool.k, sign * 1.421875 * 2.0 ** 14))
    q = torch.full((sum(q_len), 4, D), 2.0 ** 14).to(tdt(dtype))
    out = one_call(vr, pool, q, q_len, scale=2.0 ** power)
    ref, tol = mean_of(pool, q_len[0])
    within(out, ref.expand_as(out), tol.expand_as(out), "mean")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", [-13, -8, -3, 0, 1, 60, 100])
def test_attn_largest_score_takes_all(vr, dtype, form, power):
    """Scores of whole numbers (exact) times 2^20 times scale, below and beyond the largest power of two whose multiples are
    32-bit exponents: the largest that a row sees has all of the weight, several equal ones share it."""
    import torch
    q_len, kv_len, width = FORMS[form]
    m, n = q_len[0], kv_len[0]
    say(f"[largest] {dtype} {form} 2^{power}")
    pool = Pool(kv_len, 1, 32, dtype, seed=4, width=width)
    gen = torch.Generator().manual_seed(7)
    x = torch.randint(-120, 100, (n,), generator=gen)
    x[torch.randint(0, n - m, (2,), generator=gen)] = 120  # two of them before every new token
    for t in range(n):
        p, i = int(pool.table[0, t // 32]), t % 32
        pool.k[p, 0, i] = 0
        pool.k[p, 0, i, 77] = float(x[t])
    q = torch.zeros((m, 4, D))
    q[..., 77] = 2.0 ** 20
    out = one_call(vr, pool, q.to(tdt(dtype)), q_len, scale=2.0 ** power)
    ref, tol = mean_of(pool, m, x == 120)                  # the next one's weight is e^-2560 at most
    within(out, ref.expand_as(out), tol.expand_as(out), "largest")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_attn_scores_that_overflow(vr, dtype, form):
    """<q, k> beyond fp32 for the middle new token's own key: the rows that see it are NaN, those before it as they would be."""
    import torch
    q_len, kv_len, width = FORMS[form]
    m, n = q_len[0], kv_len[0]
    t = n - m + m // 2
    pool = Pool(kv_len, 1, 32, dtype, seed=5, width=width)
    q = torch.randn((m, 4, D), generator=torch.Generator().manual_seed(6)).to(tdt(dtype))
    q[..., 0] = 4.0
    ref, tol = attn_ref(pool, q, q_len, 4)
    p, i = int(pool.table[0, t // 32]), t % 32
    pool.k[p, 0, i] = 0
    pool.k[p, 0, i, 0] = 2.0 ** 127
    out = one_call(vr, pool, q, q_len)
    assert out[m // 2:].isnan().all()
    within(out[:m // 2], ref[:m // 2], tol[:m // 2], "before it")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_starts_that_fall(vr, dtype):
    """Starts 0, T, 0, T, ..: 32 sequences that all claim every row are more work than a call can have.  Nothing is computed, and
    a proper call with the same workspace is as it would be."""
    import torch
    S, T, n = 64, 300, 600
    pool = Pool([n] * S, 1, 32, dtype, seed=9)
    q = torch.randn((T, 4, D), generator=torch.Generator().manual_seed(8)).to(tdt(dtype)).cuda()
    pages, batch = pool.device(vr, [T] + [0] * (S - 1))
    bad = torch.tensor([(s & 1) * T for s in range(S + 1)], dtype=torch.int32).cuda()
    falling = vr.PagedBatch(batch.table, batch.kv_len, bad)
    ws = torch.full((96 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((T, 4, D), 5.0, dtype=tdt(dtype), device="cuda")
    say(f"[falling starts] {dtype}")
    vr.paged_attn(pages, falling, q, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert (out == 5).all()
    assert torch.equal(vr.paged_attn(pages, batch, q, workspace=ws), vr.paged_attn(pages, batch, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-6])
def test_norm_of_any_size(vr, dtype, eps):
    """Rows whose squares leave fp32's range either way are normed by the formula: beside ordinary rows, with values of
    very different sizes in a row, with and without rotation."""
    import torch
    from test_gpu_paged import norm_ref, theta_of
    gen = torch.Generator().manual_seed(4)
    powers = [-126, -100, -75, -63, -50, -40, -20, 0, 20, 50, 62, 63, 64, 65, 80, 100, 125]
    x = torch.randn((len(powers), 3, D), generator=gen).clamp(-3.5, 3.5)
    x *= 2.0 ** torch.tensor(powers, dtype=torch.float32)[:, None, None]
    x[:, 1, 1:] *= 2.0 ** -30                              # one value far above the others
    x[:, 2, ::2] = 0
    x = x.to(tdt(dtype))
    w = 1 + 0.3 * torch.randn((3, D), generator=gen)
    pos = torch.arange(len(powers), dtype=torch.int32) * 1000
    for theta in (None, theta_of()):
        say(f"[norm sizes] {dtype} eps={eps} rotated={theta is not None}")
        got, _ = vr.norm_rotate(x.cuda(), wq=w.cuda(), eps=eps, pos=pos.cuda(), theta=None if theta is None else theta.cuda())
        ref, tol = norm_ref(x, w, pos, theta, eps, dtype)
        within(got, ref, tol, "rows")
    zero, _ = vr.norm_rotate(torch.zeros((1, 1, D), dtype=tdt(dtype), device="cuda"), wq=w[0].cuda(), eps=1e-30)
    assert (zero == 0).all()


@pytest.mark.parametrize("q_len,kv_len,G,H", [([1], [2], 2, 32), ([2], [3], 1, 7), ([4], [7], 2, 8), ([1, 3], [17, 40], 1, 5),
                                              ([1], [3000], 2, 8), ([1], [1300], 1, 16), ([2, 1], [2500, 33], 2, 16)])
def test_attn_few_rows_keep_their_weights(vr, q_len, kv_len, G, H):
    """bf16 rows of up to 16 to a KV head: the weights' rounding is made good (2^-16 is left of it), so that outputs are off by
    little more than their own rounding."""
    import torch
    say(f"[weights] q {q_len} kv {kv_len} G={G} H={H}")
    assert max(q_len) * H // G <= 16
    for seed in range(3):
        pool = Pool(kv_len, G, 16, "bf16", seed=seed)
        q = torch.randn((sum(q_len), H, D), generator=torch.Generator().manual_seed(seed + 50)).bfloat16()
        q *= 0.25                                          # weights alike: none is nothing beside the others
        out = one_call(vr, pool, q, q_len)
        at = 0
        for s, m in enumerate(q_len):
            K, V, _ = pool.rows(s)
            for i in range(m):
                n = kv_len[s] - m + i + 1
                for h in range(H):
                    k, v, x = K[:n, h * G // H].double(), V[:n, h * G // H].double(), q[at + i, h].double()
                    sc, mag = (k @ x) * D ** -0.5, (k.abs() @ x.abs()) * D ** -0.5
                    w = torch.softmax(sc, 0)
                    o, A = w @ v, w @ v.abs()
                    dx = float((128 * U32 * mag + 3 * U32 * (sc.abs() + sc.abs().max())).max()) + 2 * U32
                    e = 2.0 ** -16 * (A + o.abs()) + (4 * dx + (n + 256) * U32) * A
                    tol = (e + U["bf16"] * o.abs()) * (1 + U["bf16"]) + 1e-38
                    err = (out[at + i, h] - o).abs()
                    assert (err <= tol).all(), f"seed {seed}, sequence {s}, token {i}, head {h}: {float((err / tol).max())}"
            at += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_many_calls(vr, dtype):
    """A workspace of the caller's, full of ones, serves calls of every kind one after another (tiles whole, in equal pieces and
    divided evenly, few rows and many), each as if with memory of its own; nothing behind what a call asks for is written."""
    import torch
    assert "paged_attn_workspace" in vr.__all__
    calls = []
    for q_len, kv_len in (([1], [9000]), ([1003], [3003]), ([70] + [1] * 6, [2000, 40, 700, 1300, 4000, 5000, 100]), ([1], [40]),
                          ([300, 200], [300, 200]), ([1] * 5, [100, 2000, 4000, 8000, 9000]), ([2], [700])):
        pool = Pool(kv_len, 2, 32, dtype, seed=len(calls))
        pages, batch = pool.device(vr, q_len)
        q = torch.randn((sum(q_len), 8, D), generator=torch.Generator().manual_seed(len(calls))).to(tdt(dtype)).cuda()
        calls.append((pages, batch, q, vr.paged_attn(pages, batch, q)))
    need = [vr.paged_attn_workspace(p, b, q.shape[0], 8).numel() for p, b, q, _ in calls]
    ws = torch.full((max(need) + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    for i in list(range(len(calls))) + [6, 0, 3, 2, 1]:
        pages, batch, q, want = calls[i]
        out = vr.paged_attn(pages, batch, q, workspace=ws[:need[i]])
        assert torch.equal(out, want), i
        assert (ws[max(need):] == 0xFF).all(), i
    ws.fill_(0xFF)
    pages, batch, q, want = calls[0]
    assert torch.equal(vr.paged_attn(pages, batch, q, workspace=ws[:need[0]]), want) and (ws[need[0]:] == 0xFF).all()


# ---- long tiles, and many of them: every row of the calls in paged_shapes.py -------------------------------------------

def attn_ref_all(pool, q, q_len, H, causal, window):
    """As attn_ref, every row, a sequence's rows of a KV head together, on the device in 64 bits."""
    import torch
    G, c, dtype = pool.G, D ** -0.5, pool.dtype
    Hg, u = H // G, U[dtype]
    ref, tol = (torch.zeros((sum(q_len), H, D), dtype=torch.float64) for _ in range(2))
    at, loaded = 0, None
    for s, m in enumerate(q_len):
        n = pool.kv_len[s]
        if loaded is None or len(loaded[0]) < n:
            loaded = [x.cuda() for x in pool.rows(s)]      # all sequences have the same pages
        K, V, ok = (x[:n] for x in loaded)
        p, t = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        see = ok[None].expand(m, n)
        if causal:
            see = see & (t <= p) & ((p - t < window) if window else True)
        see = see.repeat_interleave(Hg, 0)
        none = ~see.any(1, keepdim=True)
        for g in range(G):
            x = q[at:at + m, g * Hg:(g + 1) * Hg].reshape(-1, D).cuda().double()
            k, v = torch.where(ok[:, None], K[:, g].double(), 0.0), torch.where(ok[:, None], V[:, g].double(), 0.0)
            kt = k.t().contiguous()
            sc = (x @ kt * c).masked_fill(~see, -math.inf)
            w = torch.softmax(sc, 1).masked_fill(none, 0.0)
            o, A = w @ v, w @ v.abs()
            size = sc.abs().masked_fill(~see, 0.0)
            mag = (x.abs() @ kt.abs() * c).masked_fill(~see, 0.0)
            dx = (128 * U32 * mag + 3 * U32 * (size + size.max(1, keepdim=True).values)).max(1, keepdim=True).values + 2 * U32
            e = (u if dtype == "bf16" else 0) * (A + o.abs()) + (4 * dx + (see.sum(1, keepdim=True) + 256) * U32) * A
            b = (e + u * o.abs()) * (1 + u) + 1e-38
            ref[at:at + m, g * Hg:(g + 1) * Hg] = o.reshape(m, Hg, D).cpu()
            tol[at:at + m, g * Hg:(g + 1) * Hg] = b.reshape(m, Hg, D).cpu()
        at += m
    return ref, tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("i", range(7))
def test_attn_long_and_many_tiles(vr, dtype, bad, i):
    """bad: entries that name no page in the second and the third window of 1024 keys and in the last."""
    import torch
    from paged_shapes import SHAPES
    s = SHAPES[i]
    say(f"[long] {s.name} {dtype} bad={bad}")
    pool = Pool([max(s.kv_len)], s.G, s.page, dtype, seed=i)
    if bad:
        for t, entry in ((1100, -1), (2200, pool.k.shape[0]), (min(s.kv_len) - 300, -(1 << 31))):
            pool.table[0, t // s.page] = entry
    pool.table = pool.table.expand(len(s.q_len), -1).contiguous()
    pool.kv_len = list(s.kv_len)
    q = (2 * torch.randn((sum(s.q_len), s.H, D), generator=torch.Generator().manual_seed(i + 70))).to(tdt(dtype))
    pages, batch = pool.device(vr, s.q_len)
    assert batch.table.shape[1] == s.width
    out = vr.paged_attn(pages, batch, q.cuda(), causal=s.causal, window=s.window)
    torch.cuda.synchronize()
    ref, tol = attn_ref_all(pool, q, s.q_len, s.H, s.causal, s.window)
    within(out, ref, tol, s.name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_attn_sizes_of_scores_beside_each_other(vr, dtype, form):
    """One head's scores are beyond what exponents hold, from a late key on, another's hugely negative but for the last keys; the
    ordinary rows beside them in a wave are as they would be."""
    import torch
    q_len, kv_len, width = FORMS[form]
    m, n = q_len[0], kv_len[0]
    pool = Pool(kv_len, 1, 32, dtype, seed=15, width=width)
    far = n - m - 60                                       # the key that is large for head 0
    for t in range(n):
        p, i = int(pool.table[0, t // 32]), t % 32
        pool.k[p, 0, i, 100] = 2.0 ** 20 if t == far else 0
        pool.k[p, 0, i, 101] = -2.0 ** 20 if t < n - m - 20 else 0
    q = torch.randn((m, 4, D), generator=torch.Generator().manual_seed(16)).to(tdt(dtype))
    q[..., 100:102] = 0
    want = attn_ref(pool, q, q_len, 4)
    q[:, 0, 100], q[:, 1, 101] = 2.0 ** 30, 2.0 ** 30
    out = one_call(vr, pool, q, q_len)
    _, V, _ = pool.rows(0)
    assert torch.equal(out[:, 0], V[far, 0].double().expand(m, D))
    within(out[:, 2:], want[0][:, 2:], want[1][:, 2:], "beside")
    K, _, _ = pool.rows(0)
    q[:, 1, 101] = 0
    for i in range(m):                                     # head 1: the last keys alone count
        see = slice(n - m - 20, n - m + i + 1)
        k, v, x = K[see, 0].double(), V[see, 0].double(), q[i, 1].double()
        sc, mag = (k @ x) * D ** -0.5, (k.abs() @ x.abs()) * D ** -0.5
        w = torch.softmax(sc, 0)
        o, A = w @ v, w @ v.abs()
        dx = float((128 * U32 * mag + 3 * U32 * (sc.abs() + sc.abs().max())).max()) + 2 * U32
        u = U[dtype]
        e = (u if dtype == "bf16" else 0) * (A + o.abs()) + (4 * dx + (len(k) + 256) * U32) * A
        within(out[i, 1], o, (e + u * o.abs()) * (1 + u) + 1e-38, "last keys")
