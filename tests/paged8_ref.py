"""The 8-bit paged cache in 64 bits on the host: codes, pools, and the operators over them, written from their definitions."""
import math

import torch

D, B = 128, 32
E_LO, E_HI = -110, 119
U32 = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def exponent(x):
    """The exponent of the scale of rows x [..., rows, d]: infinities and NaN do not count."""
    most = torch.where(torch.isfinite(x), x.double().abs(), 0.0).amax(dim=(-2, -1))
    e = torch.full(most.shape, E_LO, dtype=torch.int32)
    while bool((more := (most > 448 * torch.exp2(e.double())) & (e < E_HI)).any()):
        e = e + more.int()
    return e


def nearest(y):
    """y (64 bits) rounded to e4m3 values, ties to even; infinities become NaN."""
    y = y.double()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(2.0 ** -6, 448.0))) - 3)
    z = (torch.round(y / step) * step).clamp(-448, 448)
    return torch.where(torch.isfinite(y), z, math.nan)


class Pool8:
    """Codes as the numbers that they stand for (64 bits, before the scale) and exponents; junk: what unused slots hold."""

    def __init__(self, kv_len, G, page, seed=0, width=None, spare=2, junk=math.nan, fill=True, kscale=1.0):
        gen = torch.Generator().manual_seed(seed)
        need = [(n + page - 1) // page for n in kv_len]
        self.total, self.G, self.page, self.kv_len = sum(need) + spare, G, page, list(kv_len)
        shape = (self.total, G, page, D)
        self.code = {x: torch.full(shape, junk, dtype=torch.float64) for x in "kv"}
        self.exp = {x: torch.full((self.total, G, page // B), 5, dtype=torch.int32) for x in "kv"}
        self.table = torch.full((len(kv_len), max(need + [1]) if width is None else width), -1, dtype=torch.int32)
        order = torch.randperm(self.total, generator=gen)
        self.free = order[sum(need):].tolist()
        at = 0
        for s, m in enumerate(need):
            self.table[s, :m] = order[at:at + m].int()
            at += m
        if fill:
            for s, n in enumerate(kv_len):
                for x in "kv":
                    rows = (kscale if x == "k" else 1.0) * torch.randn((n, G, D), generator=gen)
                    rows *= torch.exp2(torch.randint(-2, 3, (n, G, 1), generator=gen))       # blocks of unlike scales
                    self.append_rows(s, 0, rows, x)

    def good(self, s, t):
        p = int(self.table[s, t // self.page])
        return p if 0 <= p < self.total else -1

    def append_rows(self, s, t0, rows, x):
        """Rows [n][G][d] of keys or values from position t0 of sequence s on."""
        n, t = rows.shape[0], t0
        while t < t0 + n:
            m = min(B - t % B, t0 + n - t)
            p, b = self.good(s, t), t % self.page // B
            if p >= 0:
                new = rows[t - t0:t - t0 + m].transpose(0, 1).double()             # [G][m][d]
                e = exponent(new)
                c = self.code[x][p].view(self.G, -1, B, D)[:, b]
                if t % B:
                    was = self.exp[x][p][:, b]
                    e = torch.maximum(e, was)
                    again = nearest(c[:, :t % B] * torch.exp2((was - e).double())[:, None, None])
                    c[:, :t % B] = torch.where(torch.isnan(c[:, :t % B]), c[:, :t % B], again)
                c[:, t % B:t % B + m] = nearest(new * torch.exp2(-e.double())[:, None, None])
                self.exp[x][p][:, b] = e
            t += m

    def values(self, x):
        """The pool's values [pages][G][page][d]."""
        return self.code[x] * torch.exp2(self.exp[x].double()).repeat_interleave(B, dim=2)[..., None]

    def rows(self, s, n=None):
        """(K, V) [n][G][d] of sequence s, and which of them have a page."""
        n = max(self.kv_len[s], 0) if n is None else n
        t = torch.arange(n)
        pg = self.table[s][t // self.page].long()
        ok = (pg >= 0) & (pg < self.total)
        pg = torch.where(ok, pg, 0)
        f = lambda x: (self.code[x][pg, :, t % self.page]
                       * torch.exp2(self.exp[x][pg, :, t % self.page // B].double())[..., None])
        return f("k"), f("v"), ok

    def device(self, vr):
        c = {x: self.code[x].float().to(torch.float8_e4m3fn).cuda() for x in "kv"}
        e = {x: (self.exp[x] + 127).to(torch.uint8).view(torch.float8_e8m0fnu).cuda() for x in "kv"}
        return vr.PagedCache8(c["k"], c["v"], e["k"], e["v"])

    def batch(self, vr, q_len, pad=0):
        start = torch.tensor([pad + sum(q_len[:s]) for s in range(len(q_len) + 1)], dtype=torch.int32)
        return vr.PagedBatch(self.table.cuda(), torch.tensor(self.kv_len, dtype=torch.int32).cuda(), start.cuda())

    def same(self, pages):
        """The device's pool holds these codes and scales, NaN for NaN."""
        for x, c, e in (("k", pages.k, pages.k_scale), ("v", pages.v, pages.v_scale)):
            got, exps = c.cpu().float().double(), e.view(torch.uint8).cpu().int() - 127
            bad = ~((got == self.code[x]) | (torch.isnan(got) & torch.isnan(self.code[x])))
            assert torch.equal(exps, self.exp[x]), f"{x}: exponents differ at {(exps != self.exp[x]).nonzero()[:4].tolist()}"
            assert not bad.any(), f"{x}: {int(bad.sum())} codes differ, at {bad.nonzero()[:4].tolist()}"


def seen_by(n, m, causal, window):
    """[m][n]: which keys each of the last m of n tokens sees."""
    p, t = torch.arange(n - m, n)[:, None], torch.arange(n)[None, :]
    if not causal:
        return torch.ones((m, n), dtype=torch.bool)
    see = t <= p
    return see & (p - t < window) if window else see


def attn_ref(pool, q, q_len, H, dtype, causal=True, window=0, scale=None):
    """out, its bound, lse, its bound (64 bits).

    A code's value is exact.  bf16 queries: a score is 128 products summed in fp32, 128 u32 sum|q k|; fp32 queries are three
    exact parts of one sign, 384 products of the same sum of magnitudes.  The exponent's product and sum 3 u32 (|c x| +
    |c m|), the exponential 2 u32: together D.  Weights are rounded in their products with the values: u_p of A = sum p |v| /
    sum p (bf16 2^-8, at least one form; fp32 exact parts), and sums of n weighted values in up to 3 parts 3 n u32.  A weight's
    error counts in maximum and sum, so |error| <= u_p A + (4 D + (3 n + 256) u32) A, then the output's rounding.
    lse: D for every weight, n + 64 u32 for their sum, and its own terms 4 u32 (1 + |lse| + |c m|)."""
    G, c = pool.G, 1 / math.sqrt(D) if scale is None else scale
    T = sum(q_len)
    ref, tol = torch.zeros((T, H, D), dtype=torch.float64), torch.zeros((T, H, D), dtype=torch.float64)
    lse, ltol = torch.full((T, H), -math.inf, dtype=torch.float64), torch.zeros((T, H), dtype=torch.float64)
    terms = 128 if dtype == "bf16" else 384
    u = U[dtype]
    at = 0
    for s, m in enumerate(q_len):
        n = pool.kv_len[s]
        K, V, ok = pool.rows(s)
        if m and n:
            see = seen_by(n, m, causal, window) & ok
            live = see.any(-1)
            for h in range(H):
                k, v, x = K[:, h // (H // G)], V[:, h // (H // G)], q[at:at + m, h].double()
                k = torch.where(see.any(0)[:, None], k, 0.0)       # keys that nobody sees do not count, whatever they hold
                sc = torch.where(see, (x @ k.T) * c, -math.inf)
                w = torch.where(live[:, None], torch.softmax(sc, -1).nan_to_num(0.0), 0.0)
                v0 = torch.where(see.any(0)[:, None] & torch.isfinite(v), v, 0.0)
                o, A = w @ v0, w @ v0.abs()
                nan = (see.double() @ (torch.isnan(v) & see.any(0)[:, None]).double()) > 0
                z = sc.abs().masked_fill(~see, 0.0)
                dx = terms * U32 * c * ((x.abs() @ k.abs().T).masked_fill(~see, 0.0)).amax(-1) + 6 * U32 * z.amax(-1) + 2 * U32
                e = ((u if dtype == "bf16" else 0.0) + (4 * dx + (3 * n + 256) * U32))[:, None] * A
                ref[at:at + m, h] = torch.where(nan, math.nan, o)
                tol[at:at + m, h] = (e + u * o.abs()) * (1 + u) + 1e-38
                lse[at:at + m, h] = torch.where(live, torch.logsumexp(sc, -1), -math.inf)
                ltol[at:at + m, h] = 2 * dx + (n + 64) * U32 + 4 * U32 * (1 + lse[at:at + m, h].abs().nan_to_num(0.0, 0.0, 0.0) + z.amax(-1))
        at += m
    return ref, tol, lse, ltol


def mass_ref(pool, q, q_len, H, lse, mass, dtype, causal=True, window=0, scale=None):
    """What paged8_mass adds up to, and its bound: a weight's exponent is off by the score's error and by 4 u32 of what is
    subtracted (|c x| + |lse|), its exponential 2 u32, the sum of R rows R u32, and the old mass and the result u32 each."""
    G, c = pool.G, 1 / math.sqrt(D) if scale is None else scale
    out, tol = mass.double().clone(), torch.zeros(mass.shape, dtype=torch.float64)
    terms = 128 if dtype == "bf16" else 384
    L = mass.shape[2]
    at = 0
    for s, m in enumerate(q_len):
        n = min(pool.kv_len[s], L)
        N = pool.kv_len[s]
        K, _, ok = pool.rows(s)
        out[s, :, max(0, min(n, N - m)):n] = 0
        if m and n:
            see = (seen_by(N, m, causal, window) & ok)[:, :n]
            for h in range(H):
                g = h // (H // G)
                x, k = q[at:at + m, h].double(), torch.where(see.any(0)[:, None], K[:n, g], 0.0)
                z = lse[at:at + m, h].double()[:, None]
                sc = (x @ k.T) * c
                w = torch.where(see & (z > -math.inf), torch.exp(sc - z), 0.0)
                dx = terms * U32 * c * (x.abs() @ k.abs().T) + 4 * U32 * (sc.abs() + z.abs().nan_to_num(0.0, 0.0, 0.0)) + 2 * U32
                out[s, g, :n] += w.sum(0)
                tol[s, g, :n] += (w * (2 * dx + m * H * U32)).sum(0)
        at += m
        tol[s, :, :n] += 4 * U32 * out[s, :, :n].abs() + 1e-38
    return out, tol


def keep_ref(mass, n, keep, first, recent):
    """The tokens of one head that stay."""
    m = min(n, keep)
    if m == n:
        return list(range(n))
    forced = [t for t in range(n) if t < first or t >= n - recent]
    rest = [t for t in range(n) if first <= t < n - recent]
    x = mass.tolist()
    rest.sort(key=lambda t: (math.isnan(x[t]), 0.0 if math.isnan(x[t]) else -x[t], t))
    return sorted(forced + rest[:m - len(forced)])


def evict_ref(pool, table_into, mass, keep, first, recent):
    """index, mass_out, len_out; the pool changes."""
    S, G, L = mass.shape
    index, kept = torch.full((S, G, keep), -1, dtype=torch.int32), torch.zeros((S, G, keep))
    lens = torch.zeros(S, dtype=torch.int32)
    source = [pool.rows(s) for s in range(S)]
    for s in range(S):
        n = min(max(pool.kv_len[s], 0), L)
        m = lens[s] = min(n, keep)
        for g in range(G):
            stay = torch.tensor(keep_ref(mass[s, g, :n], n, keep, first, recent), dtype=torch.long)
            index[s, g, :m], kept[s, g, :m] = stay.int(), mass[s, g][stay]
            for x, rows in (("k", source[s][0]), ("v", source[s][1])):
                r = torch.where(source[s][2][stay][:, None], rows[stay, g], 0.0)
                for b in range(0, int(m), B):
                    p = int(table_into[s, b // pool.page])
                    if not 0 <= p < pool.total:
                        continue
                    y = r[b:b + B]
                    e = exponent(y)
                    at = b % pool.page
                    pool.code[x][p, g, at:at + y.shape[0]] = nearest(y * torch.exp2(-e.double()))
                    pool.exp[x][p, g, at // B] = e
    return index, kept, lens
