"""The 8-bit paged cache as it is used: strides, padding, streams, graphs, pools beyond 32 bits, scores of any size, a serving run
from the prompt to the codec, and what the binding refuses."""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

D = 128


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


def within(*a):
    from test_gpu_paged8 import within as f
    f(*a)


def copy_of(vr, pages):
    import torch
    return vr.PagedCache8(*(t.view(torch.uint8).clone().view(t.dtype) for t in (pages.k, pages.v, pages.k_scale, pages.v_scale)))


def same_pages(a, b):
    import torch
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8))
               for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)))


def queries(T, H, dtype, seed, scale=2.0):
    import paged8_ref as R
    import torch
    return (scale * torch.randn((T, H, D), generator=torch.Generator().manual_seed(seed))).to(R.tdt(dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [[2, 0, 1], [70, 0, 33]])
def test_padding_and_strides(vr, R, dtype, q_len):
    """Rows before the first sequence and behind the last are left as they were; slices of a fused projection, outputs with gaps, one
    row for all tokens (stride 0), tables and lengths that are slices."""
    import torch
    G, H, pad = 2, 6, 3
    kv = [300, 40, 133]
    pool = R.Pool8(kv, G, 32, seed=1, width=12)
    T = sum(q_len) + 2 * pad
    x = queries(T, H + 2 * G, dtype, 2).cuda()
    wide = torch.full((3, 20), -7, dtype=torch.int32, device="cuda")
    wide[:, 4:16] = pool.table.cuda()
    lens = torch.tensor([9, 9] + kv, dtype=torch.int32).cuda()[2:]
    pages = pool.device(vr)
    batch = vr.PagedBatch(wide[:, 4:16], lens, pool.batch(vr, q_len, pad).q_start)
    out = torch.full((T, H + 1, D), 7.0, dtype=x.dtype, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda")
    vr.paged8_attn(pages, batch, x[:, :H], out=out[:, :H], lse=lse)
    ref, tol, lref, ltol = R.attn_ref(pool, x[pad:T - pad, :H].cpu(), q_len, H, dtype)
    within(out[pad:T - pad, :H], ref, tol, "out")
    within(lse[pad:T - pad], lref, ltol, "lse")
    assert (out[:pad] == 7).all() and (out[T - pad:] == 7).all() and (out[:, H] == 7).all()
    assert (lse[:pad] == 7).all() and (lse[T - pad:] == 7).all()
    row = x[pad:pad + 1, :H].expand(T, H, D)
    assert torch.equal(vr.paged8_attn(pages, batch, row)[pad:T - pad], vr.paged8_attn(pages, batch, row.contiguous())[pad:T - pad])
    mass = torch.rand((3, G, 310), generator=torch.Generator().manual_seed(3))
    got = vr.paged8_mass(pages, batch, x[:, :H], lse, mass.cuda())
    want, mtol = R.mass_ref(pool, x[pad:T - pad, :H].cpu(), q_len, H, lse[pad:T - pad].cpu(), mass, dtype)
    for s, n in enumerate(kv):
        within(got[s, :, :n], want[s, :, :n], mtol[s, :, :n], f"mass {s}")
    # one row for all tokens, and rows of unlike strides
    row = x[:1, :G].expand(T, G, D)
    a, b = pool.device(vr), pool.device(vr)
    vr.paged8_append(a, batch, row, x[:, G:2 * G])
    vr.paged8_append(b, batch, row.contiguous(), x[:, G:2 * G].contiguous())
    assert same_pages(a, b) and not same_pages(a, pages)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([1], [40000]), ([1, 1, 1], [3000, 50, 9000]), ([300], [3000])])
def test_same_bits_again(vr, R, dtype, q_len, kv_len):
    """Two runs, and runs with memory of the caller's, give the same bits."""
    import torch
    pool = R.Pool8(kv_len, 2, 64, seed=3, fill=False, junk=0.0)
    pages, batch = pool.device(vr), pool.batch(vr, q_len)
    for t in (pages.k, pages.v):
        t.view(torch.uint8).copy_(torch.randint(0, 120, t.shape, dtype=torch.uint8))
    q = queries(sum(q_len), 8, dtype, 4, 1e-3).cuda()
    ws = vr.paged8_attn_workspace(pages, batch, sum(q_len), 8, q.dtype)
    runs = []
    for w in (None, None, ws, ws):
        lse = torch.empty(q.shape[:2], device="cuda")
        out = vr.paged8_attn(pages, batch, q, lse=lse, workspace=w)
        mass = vr.paged8_mass(pages, batch, q, lse, torch.zeros((len(kv_len), 2, max(kv_len)), device="cuda"))
        runs.append((out, lse, mass))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
    assert not runs[0][0].isnan().any()


def test_two_streams_at_once(vr, R):
    import torch
    pool = R.Pool8([5000, 4000], 2, 64, seed=17)
    pages, batch = pool.device(vr), pool.batch(vr, [1, 1])
    qs = [queries(2, 8, "bf16", s).cuda() for s in range(2)]

    def call(i):
        lse = torch.empty((2, 8), device="cuda")
        out = vr.paged8_attn(pages, batch, qs[i], lse=lse)
        return out, lse, vr.paged8_mass(pages, batch, qs[i], lse, torch.zeros((2, 2, 5000), device="cuda"))

    want = [call(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(8):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(call(i))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r, want[i]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps_follow_new_lengths(vr, R, dtype):
    """A serving step (append, attend, add up, evict) captured twice and replayed with new rows and lengths, eager steps between."""
    import torch
    G, H, page, S, pad, keep = 2, 8, 32, 3, 1, 40
    dt = R.tdt(dtype)
    lens = [30, 1, 700]
    pool = R.Pool8([v + 20 for v in lens], G, page, seed=7, spare=8, junk=0.0)
    pages = pool.device(vr)
    x = torch.zeros((S + pad, H + 2 * G, D), dtype=dt, device="cuda")
    kv = torch.tensor(lens, dtype=torch.int32).cuda()
    batch = vr.PagedBatch(pool.table.cuda(), kv, torch.arange(S + 1, dtype=torch.int32).cuda())
    into = torch.tensor(pool.free[:6], dtype=torch.int32).view(3, 2).cuda()

    class Run:
        def __init__(self, pages):
            self.pages = pages
            self.out = torch.zeros((S + pad, H, D), dtype=dt, device="cuda")
            self.lse = torch.zeros((S + pad, H), device="cuda")
            self.mass = torch.zeros((S, G, 730), device="cuda")
            self.index = torch.zeros((S, G, keep), dtype=torch.int32, device="cuda")
            self.kept = torch.zeros((S, G, keep), device="cuda")

        def step(self):
            vr.paged8_append(self.pages, batch, x[:, H:H + G], x[:, H + G:])
            vr.paged8_attn(self.pages, batch, x[:, :H], out=self.out, lse=self.lse)
            vr.paged8_mass(self.pages, batch, x[:, :H], self.lse, self.mass)
            index, kept, _ = vr.paged8_evict(self.pages, batch.table, kv, self.mass, keep, into, first=2, recent=8)
            self.index.copy_(index)
            self.kept.copy_(kept)

    eager, caught = Run(copy_of(vr, pages)), Run(pages)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        Run(copy_of(vr, pages)).step()
    side.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            caught.step()
        graphs.append(g)
    gen = torch.Generator().manual_seed(31)
    for i in range(6):
        kv.copy_(torch.tensor([v + i + 1 for v in lens], dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=gen).to(dt))
        graphs[i % 2].replay()
        got = [t.clone() for t in (caught.out[:S], caught.lse[:S], caught.mass, caught.index, caught.kept)]
        eager.step()
        torch.cuda.synchronize()
        for a, b in zip(got, (eager.out[:S], eager.lse[:S], eager.mass, eager.index, eager.kept)):
            assert torch.equal(a, b), i
        assert same_pages(caught.pages, eager.pages), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(vr, R, dtype):
    """The same sequence in a small pool and at the end of one whose codes take more than 2^32 bytes."""
    import torch
    G, H, page, n = 8, 16, 256, 700
    far = (1 << 32) // (G * page * D) + 40
    small = R.Pool8([n], G, page, seed=5, spare=3)
    a = small.device(vr)
    big = vr.PagedCache8(*(torch.empty((far,) + shape, dtype=torch.uint8, device="cuda").view(t)
                           for shape, t in (((G, page, D), torch.float8_e4m3fn), ((G, page, D), torch.float8_e4m3fn),
                                            ((G, page // 32), torch.float8_e8m0fnu), ((G, page // 32), torch.float8_e8m0fnu))))
    shift = far - a.k.shape[0]
    u8 = lambda t: t.view(torch.uint8)
    for x, y in zip((big.k, big.v, big.k_scale, big.v_scale), (a.k, a.v, a.k_scale, a.v_scale)):
        u8(x)[shift:] = u8(y)
    q = queries(3, H, dtype, 6).cuda()
    k = queries(3, G, dtype, 7).cuda()
    runs = []
    for pages, off in ((a, 0), (big, shift)):
        batch = vr.PagedBatch((small.table + off).cuda(), torch.tensor([n], dtype=torch.int32).cuda(), torch.tensor([0, 3], dtype=torch.int32).cuda())
        vr.paged8_append(pages, batch, k, 2 * k)
        lse = torch.empty((3, H), device="cuda")
        out = vr.paged8_attn(pages, batch, q, lse=lse)
        mass = vr.paged8_mass(pages, batch, q, lse, torch.zeros((1, G, n), device="cuda"))
        into = (torch.tensor(small.free[:2], dtype=torch.int32) + off).view(1, 2).cuda()
        index, kept, m = vr.paged8_evict(pages, batch.table, batch.kv_len, mass, 300, into, first=1, recent=9)
        runs.append((out, lse, mass, index, kept, m, *vr.paged8_gather(pages, into[0], 300, dtype=q.dtype),
                     *vr.paged8_gather(pages, batch.table[0], n, dtype=q.dtype)))
    for x, y in zip(*runs):
        assert torch.equal(x, y)
    assert runs[0][-1].abs().sum() > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 5, 12, 70])
def test_scores_beyond_exponents(vr, R, dtype, m):
    """Scores so large that the largest takes all, whichever row it is in; and ordinary rows beside them."""
    import torch
    n, G, H = 200, 1, 4
    pool = R.Pool8([n], G, 32, seed=m)
    for t in range(n):                                     # dim 100: one key alone
        p = int(pool.table[0, t // 32])
        pool.code["k"][p, 0, t % 32, 100] = 32.0 if t == 40 else 0.0
    q = queries(m, H, dtype, 1)
    q[..., 100] = 0
    want = R.attn_ref(pool, q, [m], H, dtype)
    q[:, 0, 100] = 2.0 ** 60
    lse = torch.empty((m, H), device="cuda")
    out = vr.paged8_attn(pool.device(vr), pool.batch(vr, [m]), q.cuda(), lse=lse).cpu()
    K, V, _ = pool.rows(0)
    assert torch.equal(out[:, 0].double(), V[40, 0].expand(m, D).to(out.dtype).double())
    top = float(K[40, 0, 100]) * 2.0 ** 60 / math.sqrt(D)
    assert (lse[:, 0].double().cpu() / top - 1).abs().max() < 2.0 ** -21
    within(out[:, 1:], want[0][:, 1:], want[1][:, 1:], "beside")
    within(lse[:, 1:], want[2][:, 1:], want[3][:, 1:], "lse beside")


def test_starts_that_fall_end(vr, R):
    """Starts that fall leave outputs unspecified; the calls end and write nothing outside."""
    import torch
    S, T, G, H = 600, 64, 1, 2
    pool = R.Pool8([40], G, 32, seed=1)
    pages = pool.device(vr)
    table = pool.table.expand(S, -1).contiguous().cuda()
    start = torch.tensor([0, T] * (S // 2) + [0], dtype=torch.int32).cuda()
    batch = vr.PagedBatch(table, torch.full((S,), 40, dtype=torch.int32).cuda(), start)
    q = queries(T, H, "bf16", 2).cuda()
    vr.paged8_append(pages, batch, q[:, :1].contiguous(), q[:, 1:].contiguous())
    vr.paged8_attn(pages, batch, q)
    out = torch.full((S + 1, G, 50), 3.0, device="cuda")
    vr.paged8_mass(pages, batch, q, torch.zeros((T, H), device="cuda"), torch.zeros((S, G, 50), device="cuda"), out=out[:S])
    torch.cuda.synchronize()
    assert (out[S] == 3).all() and (out[:, :, 40:] == 3).all()


def test_attn_many_heads_and_sequences(vr, R):
    """More rows of one token than a tile of few holds, more sequences than one look takes, and odd heads."""
    from test_gpu_paged8 import check_attn, check_mass
    check_attn(vr, R, [1, 2], [300, 77], 1, 300, 32, "bf16", seed=1)
    check_attn(vr, R, [1, 2], [300, 77], 1, 70, 32, "f32", seed=2)
    kv = [1 + (97 * s) % 150 for s in range(1000)]
    check_attn(vr, R, [1] * 1000, kv, 1, 2, 32, "bf16", seed=3)
    check_mass(vr, R, [1, 2], [300, 77], 1, 300, 32, "bf16", seed=4)
    check_mass(vr, R, [1] * 1000, kv, 1, 2, 32, "f32", seed=5)


def test_evict_longer_than_one_part(vr, R):
    """More tokens than a selection holds at once: against torch's stable order, ties over the border among them."""
    import torch
    n, G, keep = 70001, 2, 9000
    gen = torch.Generator().manual_seed(1)
    mass = torch.rand((1, G, n + 3), generator=gen) ** 6
    mass[0, 1] = torch.randint(0, 9, (n + 3,), generator=gen).float()
    pages = vr.new_pages8((n + keep) // 256 + 3, G, 256)
    for t in (pages.k, pages.v):
        t.view(torch.uint8).copy_(torch.randint(0, 127, t.shape, generator=gen, dtype=torch.uint8))
    need = (n + 255) // 256
    table = torch.arange(need, dtype=torch.int32).view(1, -1).cuda()
    into = (need + torch.arange((keep + 255) // 256, dtype=torch.int32)).view(1, -1).cuda()
    kv = torch.tensor([n], dtype=torch.int32).cuda()
    index, kept, m = vr.paged8_evict(pages, table, kv, mass.cuda(), keep, into, first=5, recent=100)
    assert m.tolist() == [keep]
    w = mass[0, :, :n].clone()
    w[:, :5] = w[:, n - 100:] = math.inf
    want = torch.sort(torch.sort(w, dim=-1, descending=True, stable=True).indices[:, :keep], dim=-1).values
    assert torch.equal(index[0].cpu().long(), want)
    assert torch.equal(kept[0].cpu(), mass[0, :, :n].gather(1, want))
    K, V = vr.paged8_gather(pages, table[0], n, dtype=torch.float32)
    k2, v2 = vr.paged8_gather(pages, into[0], keep, dtype=torch.float32)
    for x, y in ((K, k2), (V, v2)):
        for g in range(G):
            src = x[want[g].cuda(), g].view(-1, D)
            assert torch.equal(y[:, g], src)               # all blocks had one scale, and none gets a larger one


@pytest.mark.parametrize("n,keep,first,recent", [(32769, 32768, 0, 1), (65536, 1, 0, 0), (65536, 40000, 3, 33000), (98305, 65537, 0, 7), (98305, 5000, 4, 0)])
def test_evict_parts_and_masses(vr, n, keep, first, recent):
    """Long sequences whose masses are equal, all but equal, NaN beyond some, and decided by a leading digit, beside a short one."""
    import torch
    G = 4
    gen = torch.Generator().manual_seed(n + keep)
    mass = torch.zeros((2, G, n))
    mass[0, 0] = 0.25                                          # one value
    mass[0, 1] = 1.0 + torch.randint(0, 3, (n,), generator=gen) * 2.0 ** -23   # apart in the last digit only
    mass[0, 2] = float("nan")
    mass[0, 2, torch.randperm(n, generator=gen)[: n // 5]] = 2.0
    mass[0, 3, torch.randperm(n, generator=gen)[:keep]] = 3.0  # exactly `keep` of them, but for the first and recent ones
    mass[1] = torch.rand((G, n), generator=gen)
    kv = [n, 3000]
    pages = vr.new_pages8((n + 3000 + 2 * keep) // 256 + 8, G, 256)
    need, into_w = (n + 255) // 256, (keep + 255) // 256
    table = torch.full((2, need), -1, dtype=torch.int32)
    table[0] = torch.arange(need)
    table[1, :12] = need + torch.arange(12)
    into = need + 12 + torch.arange(into_w, dtype=torch.int32)
    into = torch.stack([into, into + into_w])
    index, kept, m = vr.paged8_evict(pages, table.cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), mass.cuda(), keep, into.cuda(),
                                     first=first, recent=recent)
    assert m.tolist() == [min(k, keep) for k in kv]
    for s, k in enumerate(kv):
        left = min(k, keep)
        for g in range(G):
            w = mass[s, g, :k].double()
            w = torch.where(torch.isnan(w), -math.inf, w)
            w[:first] = w[max(0, k - recent):] = math.inf
            want = torch.sort(torch.sort(w, descending=True, stable=True).indices[:left]).values
            assert torch.equal(index[s, g, :left].cpu().long(), want), (s, g)
            assert torch.equal(kept[s, g, :left].cpu().nan_to_num(-1.0), mass[s, g, want].nan_to_num(-1.0)), (s, g)
            assert bool((index[s, g, left:] == -1).all()) and bool((kept[s, g, left:] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_serving_run(vr, R, dtype):
    """A prompt in chunks, single tokens, an eviction, more tokens on the evicted cache, and the hand-over to the codec."""
    import torch
    G, H, page = 2, 8, 32
    dt = R.tdt(dtype)
    n0, steps, keep, more = 500, 3, 200, 4
    total = n0 + steps
    pool = R.Pool8([total], G, page, seed=1, width=20, spare=10, fill=False, junk=0.0)
    pages = pool.device(vr)
    mass = torch.zeros((1, G, 640), device="cuda")
    mref = torch.zeros((1, G, 640), dtype=torch.float64)
    mtol = torch.zeros((1, G, 640), dtype=torch.float64)
    at = 0
    for i, m in enumerate([300, 200] + [1] * steps):
        k, v = queries(m, G, dtype, 10 + i, 1.0), queries(m, G, dtype, 30 + i, 1.0)
        q = queries(m, H, dtype, 50 + i)
        for x, rows in (("k", k), ("v", v)):
            pool.append_rows(0, at, rows, x)
        at += m
        pool.kv_len = [at]
        batch = pool.batch(vr, [m])
        vr.paged8_append(pages, batch, k.cuda(), v.cuda())
        lse = torch.empty((m, H), device="cuda")
        out = vr.paged8_attn(pages, batch, q.cuda(), lse=lse)
        ref, tol, lref, ltol = R.attn_ref(pool, q, [m], H, dtype)
        within(out, ref, tol, f"out {i}")
        within(lse, lref, ltol, f"lse {i}")
        vr.paged8_mass(pages, batch, q.cuda(), lse, mass)
        mref, t = R.mass_ref(pool, q, [m], H, lse.cpu(), mref, dtype)
        mtol = mtol + t
        within(mass[:, :, :at], mref[:, :, :at], mtol[:, :, :at], f"mass {i}")
    pool.same(pages)
    # the weights of a row add up to 1: each head's mass to the rows it was paid by
    rows = (H // G) * total
    assert (mass[0, :, :total].double().sum(-1) - rows).abs().max() < rows * (2.0 ** -12)
    into = torch.tensor(pool.free[:8], dtype=torch.int32).view(1, 8)
    index, mass2, kv = vr.paged8_evict(pages, pool.batch(vr, [0]).table, torch.tensor([total], dtype=torch.int32).cuda(), mass, keep,
                                       into.cuda(), first=4, recent=32)
    want = R.evict_ref(pool, into, mass.cpu(), keep, 4, 32)
    assert torch.equal(index.cpu(), want[0]) and torch.equal(mass2.cpu(), want[1]) and kv.tolist() == [keep]
    pool.same(pages)
    pool.table, at = into, keep
    mass = torch.zeros((1, G, 256), device="cuda")
    mass[:, :, :keep] = mass2
    for i in range(more):
        k, v, q = queries(1, G, dtype, 70 + i, 1.0), queries(1, G, dtype, 80 + i, 1.0), queries(1, H, dtype, 90 + i)
        for x, rows in (("k", k), ("v", v)):
            pool.append_rows(0, at, rows, x)
        at += 1
        pool.kv_len = [at]
        batch = pool.batch(vr, [1])
        vr.paged8_append(pages, batch, k.cuda(), v.cuda())
        out = vr.paged8_attn(pages, batch, q.cuda())
        ref, tol, _, _ = R.attn_ref(pool, q, [1], H, dtype)
        within(out, ref, tol, f"after {i}")
    pool.same(pages)
    K, V = vr.paged8_gather(pages, into[0].cuda(), at, dtype=dt)
    k, v, _ = pool.rows(0)
    assert torch.equal(K.cpu().double(), k) and torch.equal(V.cpu().double(), v)
    # the codec takes them as they are
    shape = vr.Shape(n=at, G=G, H=H, w=32, r_min=16, kappa_pct=60, dtype=dtype)
    P = torch.linalg.qr(torch.randn((G, D, D), generator=torch.Generator().manual_seed(5)))[0].cuda().contiguous()
    Qw = queries(32, H, dtype, 99, 1.0).cuda()
    cache = vr.compress(shape, K, V, Qw, P, P)
    o = vr.decode(shape, [cache], queries(1, H, dtype, 98, 1.0).cuda(), P, P)
    assert torch.isfinite(o.float()).all()


def test_binding_refuses(vr, R):
    import torch
    pool = R.Pool8([100], 2, 32, seed=1)
    pages, batch = pool.device(vr), pool.batch(vr, [3])
    q = queries(3, 8, "bf16", 1).cuda()
    lse = torch.empty((3, 8), device="cuda")
    mass = torch.zeros((1, 2, 100), device="cuda")
    kv, table = batch.kv_len, batch.table
    into = table.clone()
    bad = [
        lambda: vr.paged8_append(pages, batch, q[:, :2].half(), q[:, :2].half()),
        lambda: vr.paged8_append(pages, batch, q[:, :2], q[:, :2].float()),
        lambda: vr.paged8_append(pages, batch, q[:, :3], q[:, :3]),
        lambda: vr.paged8_append(pages, batch, q[:, :2], q[:2, :2]),
        lambda: vr.paged8_append(pages, batch, q[:, :2].cpu(), q[:, :2].cpu()),
        lambda: vr.paged8_append(pages, batch, q[:, :2, :64], q[:, :2, :64]),
        lambda: vr.paged8_attn(pages, batch, q[:, :7]),
        lambda: vr.paged8_attn(pages, batch, q, out=q),
        lambda: vr.paged8_attn(pages, batch, q, out=q.float()),
        lambda: vr.paged8_attn(pages, batch, q, lse=lse[:2]),
        lambda: vr.paged8_attn(pages, batch, q, lse=lse.double()),
        lambda: vr.paged8_attn(pages, batch, q, lse=lse.cpu()),
        lambda: vr.paged8_attn(pages, batch, q, window=(1 << 32) + 5),
        lambda: vr.paged8_attn(pages, batch, q, causal=False, window=4),
        lambda: vr.paged8_attn(pages, batch, q, scale=0.0),
        lambda: vr.paged8_attn(pages, batch, q.half()),
        lambda: vr.paged8_attn(pages, batch, q, workspace=torch.empty(8)),
        lambda: vr.paged8_attn_workspace(pages, batch, 3, 8, dtype=torch.float16),
        lambda: vr.paged8_mass(pages, batch, q, None, mass),
        lambda: vr.paged8_mass(pages, batch, q, lse[:, :4], mass),
        lambda: vr.paged8_mass(pages, batch, q, lse, mass[:, :1]),
        lambda: vr.paged8_mass(pages, batch, q, lse, mass.double()),
        lambda: vr.paged8_mass(pages, batch, q, lse, mass, out=mass[:, :, :50].contiguous()),
        lambda: vr.paged8_mass(pages, batch, q, lse, mass[:, :, ::2]),
        lambda: vr.paged8_mass(pages, batch, q, lse, mass[:, :, :0].contiguous()),
        lambda: vr.paged8_evict(pages, table, kv, mass, 0, into),
        lambda: vr.paged8_evict(pages, table, kv, mass, -3, into),
        lambda: vr.paged8_evict(pages, table, kv, mass, 1000, into),
        lambda: vr.paged8_evict(pages, table, kv, mass, 10, into, first=6, recent=5),
        lambda: vr.paged8_evict(pages, table, kv, mass, 10, into, first=-1),
        lambda: vr.paged8_evict(pages, table, kv, mass, 1 << 33, into),
        lambda: vr.paged8_evict(pages, table, kv, mass[:0], 10, into),
        lambda: vr.paged8_evict(pages, table, kv.long(), mass, 10, into),
        lambda: vr.paged8_evict(pages, table, kv, mass, 10, into[0]),
        lambda: vr.paged8_evict(pages, table, kv, mass, 10, into.cpu()),
        lambda: vr.paged8_gather(pages, table[0], -1),
        lambda: vr.paged8_gather(pages, table[0], 1000),
        lambda: vr.paged8_gather(pages, table, 10),
        lambda: vr.paged8_gather(pages, table[0], 10, dtype=torch.float16),
        lambda: vr.paged8_gather(pages, table[0], 10, K=torch.empty((10, 2, D), device="cuda")),
        lambda: vr.paged8_gather(pages, table[0], (1 << 32) + 1),
        lambda: vr.PagedCache8(pages.k, pages.v, pages.k_scale, pages.v_scale.cpu()),
        lambda: vr.new_pages8(2, 1, 16),
        lambda: vr.new_pages8(2, 1, 48),
    ]
    for i, f in enumerate(bad):
        try:
            r = f()
        except vr.VarRateError:
            continue
        if isinstance(r, vr.PagedCache8):                  # an odd page is refused by the first call
            with pytest.raises(vr.VarRateError):
                vr.paged8_gather(r, table[0], 1)
            continue
        pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
