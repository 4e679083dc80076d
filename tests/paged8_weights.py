"""Attention of few rows whose outputs show what its weights lack: few keys count, their weights are alike, and the values are 1 and -1 in
every pattern, so that in many of the 128 dims little is left of the sum and its own rounding hides nothing."""
import math

import torch

D, U32 = 128, 2.0 ** -24
LIVE = 33                                                  # keys that count, at most


def case(n, m, H, dtype):
    """(pool, q, live): one sequence of n tokens, m of them new; all keys but `live` have weights of exactly 0 (scores below -1000)."""
    import paged8_ref as R
    gen = torch.Generator().manual_seed(100 * n + m + H)
    pool = R.Pool8([n], 1, 32, 1, fill=False, junk=0.0)
    live = torch.randperm(n - m + 1, generator=gen)[:LIVE].sort().values
    k = (0.25 * torch.randn((n, 1, D), generator=gen)).clamp(-1.5, 1.5)
    k[:, 0, 100] = -28.0                                   # (one block's scale: codes of 1/64 steps and more)
    k[live, 0, 100] = 0.0
    v = torch.randint(0, 2, (n, 1, D), generator=gen).float() * 2 - 1
    pool.append_rows(0, 0, k, "k")
    pool.append_rows(0, 0, v, "v")
    q = (0.5 * torch.randn((m, H, D), generator=gen)).to(R.tdt(dtype))
    q[..., 100] = 512.0
    return pool, q, live


def weights(pool, q, live):
    """The weights of the keys that count, [m][H][live], the exact outputs, and an exponent's error: 128 products (fp32 queries: of three
    parts each) and their sum in fp32, the exponent's product and sum 3 u32 (|c x| + |c m|), the exponential 2 u32."""
    K, V, _ = pool.rows(0)
    k, v, x = K[live, 0], V[live, 0], q.double()
    sc = x @ k.T / math.sqrt(D)
    terms = 128 if q.dtype == torch.bfloat16 else 384
    mag = (x.abs() @ k.abs().T / math.sqrt(D)).amax(-1)
    dx = terms * U32 * mag + 6 * U32 * sc.abs().amax(-1) + 2 * U32
    return torch.softmax(sc, -1), v, dx


def bounds(pool, q, live, m, H, dtype):
    """out and its bound.  A = sum p |v| = 1.  bf16: a weight is its rounding and that one's rest, rounded: off by 2^-17 of it.  fp32: exact
    parts, of which the last may be cut off below 2^-24.  Sums of the products of two (three) parts, (3 live + 64) u32: keys of weight 0 add
    exact zeros, and 8 waves' (32 pieces') sums are joined.  The exponents' errors count in the weights and in their sum.  Then the output's rounding."""
    w, v, dx = weights(pool, q, live)
    o = w @ v
    e = (2.0 ** -17 if dtype == "bf16" else 2.0 ** -24) + 4 * dx + (3 * live.numel() + 64) * U32
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return o, e[..., None] * (1 + u) + u * o.abs()
