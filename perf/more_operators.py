"""Serving from a cache held in 8 bits: append new tokens' rows, attend over them, add up the weight that each
cached key is paid, evict the keys that are paid least, and hand a sequence's rows to the codec.

A pool holds keys and values as e4m3 codes [n_pages][G][page][d] and one power of two for each block of 32 tokens
and head, [n_pages][G][page / 32]: a value is its code times its block's scale.  A block's scale is the smallest
2^e, -110 <= e <= 119, that takes its largest magnitude to 448 or less (values beyond 448 x 2^119 are held as
that).  Rows appended to a block that holds some already may raise it: the codes there are rounded to the new one.

Each case is one call of one operator.  Where `own` is false the operators are computed from elementary torch
operations in 32 bits, rounded once at the end; where it is true, by the package's entry points.  Head geometries
are those of the repository's workloads: Llama (8 KV heads, 32 query heads), Qwen (4 and 28) and the tiny one
(1 and 2), head dimension 128.
"""
import math

import torch

own = False

D = 128
B = 32                                   # tokens of a block
E_LO, E_HI = -110, 119                   # exponents of a scale
HEADS = {"tiny": (1, 2), "qwen": (4, 28), "llama": (8, 32)}


def _text(lengths):
    return ",".join(str(n) for n in lengths)


def _lengths(case):
    """(new tokens, cached tokens with them) of every sequence."""
    return tuple([int(n) for n in case[k].split(",")] for k in ("q_len", "kv_len"))


def _append(heads, q_len, kv_len, *, page=64, dtype="bf16", fused=True):
    """q_len[s] new tokens at the end of kv_len[s] cached ones; fused: the rows are slices of one projection
    [T][(H + 2 G) d]."""
    return {"op": "append", "heads": heads, "q_len": _text(q_len), "kv_len": _text(kv_len), "page": page,
            "dtype": dtype, "fused": fused}


def _attn(heads, q_len, kv_len, *, page=64, dtype="bf16", causal=True, window=0, lse=False):
    """lse: the logarithm of each row's sum is wanted too."""
    return {"op": "attn", "heads": heads, "q_len": _text(q_len), "kv_len": _text(kv_len), "page": page,
            "dtype": dtype, "causal": causal, "window": window, "lse": lse}


def _mass(heads, q_len, kv_len, *, page=64, dtype="bf16"):
    return {"op": "mass", "heads": heads, "q_len": _text(q_len), "kv_len": _text(kv_len), "page": page, "dtype": dtype}


def _evict(heads, kv_len, keep, *, first=4, recent=32, page=64):
    """Of kv_len[s] tokens at most `keep` stay: the first and the most recent ones, and those of the largest mass."""
    return {"op": "evict", "heads": heads, "kv_len": _text(kv_len), "keep": keep, "first": first, "recent": recent,
            "page": page}


def _gather(heads, n, *, page=64, dtype="bf16"):
    return {"op": "gather", "heads": heads, "n": n, "page": page, "dtype": dtype}


def listed():
    cases = {
        # one decode step of 64 sequences of unlike lengths
        "append8_step_b64": _append("llama", [1] * 64, [17 + 509 * s for s in range(64)], page=32),
        # a whole prompt written at once
        "append8_llama_32k": _append("llama", [32768], [32768]),
        # the smallest attention: fp32 queries, one KV head, 512 tokens
        "attn8_step_tiny_f32": _attn("tiny", [1], [512], dtype="f32"),
        # one decode step of a long sequence, for which 8 bits are taken in the first place
        "attn8_step_llama_128k": _attn("llama", [1], [131072], lse=True),
        # chunked prefill: the last 2048 tokens of a 32768-token prompt
        "attn8_chunk_llama_32k": _attn("llama", [2048], [32768]),
        # a serving step: one odd chunk beside 16 sequences that decode
        "attn8_mixed_b17": _attn("llama", [1003] + [1] * 16, [5003] + [301 + 523 * s for s in range(16)], page=32, lse=True),
        # weights of one decode step of a batch
        "mass8_step_qwen_16k_b8": _mass("qwen", [1] * 8, [16384] * 8),
        # weights that the observation window at the end of a prompt pays it
        "mass8_window_llama_32k": _mass("llama", [32], [32768]),
        # three sequences of unlike lengths, one shorter than what may stay
        "evict8_qwen_b3": _evict("qwen", [9001, 40, 2777], 1024, page=32),
        # a prompt cut to a fifth
        "evict8_llama_32k": _evict("llama", [32768], 6554),
        # a short sequence of odd length handed to an fp32 layer's codec
        "gather8_777_f32": _gather("llama", 777, page=32, dtype="f32"),
        # the headline prompt handed to the codec
        "gather8_llama_32k": _gather("llama", 32768),
    }
    return [dict(c, name=k) for k, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "attn", "mass", "evict", "gather"])
    heads = rng.choice(["llama", "llama", "qwen", "qwen", "tiny"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([32, 64, 128, 256])
    if op == "gather":
        return _gather(heads, _log(rng, 1, 16384 if dtype == "f32" else 32768), page=page, dtype=dtype)
    if op == "append":
        S = rng.choice([1, 1, 3, 16, 64])
        q_len = [_log(rng, 1, 16384 // S) if rng.random() < 0.5 else 1 for _ in range(S)]
        kv_len = [q + rng.choice([0, _log(rng, 1, 16384 // S)]) for q in q_len]
        return _append(heads, q_len, kv_len, page=page, dtype=dtype, fused=rng.random() < 0.6)
    if op == "mass":
        if rng.random() < 0.5:
            S = rng.choice([1, 3, 8, 16])
            kv_len = [_log(rng, 1, 65536 // S) for _ in range(S)]
            return _mass(heads, [rng.choice([1, 1, min(k, 3)]) for k in kv_len], kv_len, page=page, dtype=dtype)
        q_len = [_log(rng, 8, 1024) for _ in range(rng.choice([1, 1, 2]))]
        return _mass(heads, q_len, [q + rng.choice([0, _log(rng, 1, 16384)]) for q in q_len], page=page, dtype=dtype)
    if op == "evict":
        S = rng.choice([1, 1, 4, 16])
        kv_len = [_log(rng, 1, 65536 // S) for _ in range(S)]
        keep = _log(rng, 1, max(kv_len))
        first = min(rng.choice([0, 1, 4]), keep)
        return _evict(heads, kv_len, keep, first=first, recent=min(rng.choice([0, 1, 32, 100]), keep - first), page=page)
    kind = rng.choice(["step", "step", "chunk", "prompt", "mixed"])
    window = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
    causal = True
    if kind == "step":
        S = rng.choice([1, 1, 4, 16])
        kv_len = [_log(rng, 1, (32768 if dtype == "f32" else 131072) // S) for _ in range(S)]
        q_len = [rng.choice([1, 1, 1, min(k, 4)]) for k in kv_len]
    elif kind == "chunk":
        q_len = [_log(rng, 16, 1024)]
        kv_len = [q_len[0] + _log(rng, 1, 16384)]
        causal = rng.random() < 0.8
    elif kind == "prompt":
        q_len = [_log(rng, 64, 2048) for _ in range(rng.choice([1, 2, 4]))]
        kv_len = list(q_len)
    else:
        q_len = [_log(rng, 64, 1024)] + [1] * rng.choice([3, 8])
        kv_len = [q + _log(rng, 1, 8192) for q in q_len]
    return _attn(heads, q_len, kv_len, page=page, dtype=dtype, causal=causal, window=window if causal else 0,
                 lse=rng.random() < 0.5)


# ---- inputs ------------------------------------------------------------------------------

def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _keys(gen, shape, u):
    """Keys whose channels decay, two outlier channels, 5% of the tokens planted along u."""
    sk = (1.0 / torch.arange(1, D + 1, dtype=torch.float32, device="cuda")).sqrt()
    sk[1:3] = 4.0
    k = torch.randn(shape, generator=gen, device="cuda") * sk
    hit = torch.rand(shape[:-1], generator=gen, device="cuda")
    return k + torch.where(hit < 0.05, 4.0 + 40.0 * hit, 0.0)[..., None] * u


def _exponent(amax):
    """The exponent of the scale of values up to amax."""
    m, e = torch.frexp(amax)                                   # amax = m 2^e, 1/2 <= m < 1; 448 = 7/8 x 2^9
    return torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), E_LO).clamp(E_LO, E_HI)


def _code(x, e):
    """e4m3 codes (as bytes) of x over 2^e."""
    y = torch.ldexp(x, -e).clamp(-448.0, 448.0)
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _value(code, e):
    return torch.ldexp(code.view(torch.float8_e4m3fn).float(), e)


def _pool(case, gen, need, u, filled):
    """A pool of pages in shuffled order, some of them nobody's, and page tables of need[i][s] tokens."""
    G, _ = HEADS[case["heads"]]
    P = case["page"]
    total = sum((n + P - 1) // P for row in need for n in row) + 3
    st = {}
    for name in ("k", "v"):
        shape = (total, G, P // B, B, D)
        if filled:
            x = _keys(gen, shape, u[:, None, None, :]) if name == "k" else torch.randn(shape, generator=gen, device="cuda")
            e = _exponent(x.abs().amax(dim=(-2, -1)))
            st[name] = _code(x, e[..., None, None]).view(total, G, P, D).view(torch.float8_e4m3fn)
            st[name + "_scale"] = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
            del x
        else:
            st[name] = torch.zeros((total, G, P, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            st[name + "_scale"] = torch.full((total, G, P // B), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    tables, at = [], 0
    for row in need:
        table = torch.full((len(row), max((n + P - 1) // P for n in row) + 1), -1, dtype=torch.int32, device="cuda")
        for s, n in enumerate(row):
            m = (n + P - 1) // P
            table[s, :m] = order[at:at + m]
            at += m
        tables.append(table)
    return st, tables


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    G, H = HEADS[case["heads"]]
    op = case["op"]
    u = torch.randn((G, D), generator=gen, device="cuda")
    u = u / u.norm(dim=1, keepdim=True)
    if op == "gather":
        st, (st_table,) = _pool(case, gen, [[case["n"]]], u, True)
        st.update(case=case, table=st_table)
    elif op == "evict":
        kv_len = [int(n) for n in case["kv_len"].split(",")]
        st, (table, into) = _pool(case, gen, [kv_len, [case["keep"]] * len(kv_len)], u, True)
        st.update(case=case, table=table, into=into, kv_len=torch.tensor(kv_len, dtype=torch.int32, device="cuda"))
        m = torch.rand((len(kv_len), G, max(kv_len) + 5), generator=gen, device="cuda")
        st["mass"] = torch.where(m < 0.1, 0.0, m ** 8)          # few keys hold most of it, some none
    else:
        q_len, kv_len = _lengths(case)
        T = sum(q_len)
        # an append finds the rows before it in place: of a whole prompt there are none
        filled = op != "append" or max(kv_len) > max(q_len)
        st, (table,) = _pool(case, gen, [kv_len], u, filled)
        st.update(case=case, table=table, kv_len=torch.tensor(kv_len, dtype=torch.int32, device="cuda"),
                  q_start=torch.tensor([sum(q_len[:s]) for s in range(len(q_len) + 1)], dtype=torch.int32, device="cuda"))
        if op == "append":
            k = _keys(gen, (T, G, D), u).to(_dt(case))
            v = torch.randn((T, G, D), generator=gen, device="cuda").to(_dt(case))
            if case["fused"]:
                x = torch.zeros((T, H + 2 * G, D), dtype=_dt(case), device="cuda")
                x[:, H:H + G], x[:, H + G:] = k, v
                k, v = x[:, H:H + G], x[:, H + G:]
            st["k_new"], st["v_new"] = k, v
        else:
            heads = torch.arange(H, device="cuda") // (H // G)
            q = math.sqrt(D) * u[heads] + 0.5 * torch.randn((T, H, D), generator=gen, device="cuda")
            st["q"] = q.to(_dt(case))
        if op == "mass":
            st["lse"] = _attend(st, True, 0)[1]
            st["mass"] = torch.rand((len(kv_len), G, max(kv_len) + 5), generator=gen, device="cuda")
            st["out"] = torch.zeros_like(st["mass"])
    if own:
        import paper_2607_15498_amd as vr
        st["pages"] = vr.PagedCache8(st["k"], st["v"], st["k_scale"], st["v_scale"])
        if op in ("append", "attn", "mass"):
            st["batch"] = vr.PagedBatch(st["table"], st["kv_len"], st["q_start"])
    return st


# ---- the operators -------------------------------------------------------------------------

def _bytes(st):
    return {n: st[n].view(torch.uint8) for n in ("k", "v", "k_scale", "v_scale")}


def _plain_append(st):
    P, start, kv = st["case"]["page"], st["q_start"].long(), st["kv_len"].long()
    T, pool = st["k_new"].shape[0], _bytes(st)
    i = torch.arange(T, device="cuda")
    s = torch.searchsorted(start[1:], i, right=True)           # the token's sequence
    t0 = kv - (start[1:] - start[:-1])                         # first new position of each sequence
    t = t0[s] + i - start[s]                                   # and the token's position there
    page, slot = st["table"][s, t // P].long(), t % P
    run = torch.cumsum((t % B == 0) | (t == t0[s]), 0) - 1     # the block that it falls into, counted over the call
    # blocks that hold rows already: at most the first of every sequence
    old_page, old_block = st["table"].gather(1, (t0 // P)[:, None])[:, 0].long().clamp(min=0), t0 % P // B
    held = (torch.arange(B, device="cuda")[None, :] < (t0 % B)[:, None])[:, None, :, None]      # [S][1][32][1]
    some = (t0 % B > 0)[:, None]
    first_run = run[start[:-1]]
    for name in ("k", "v"):
        x = st[name + "_new"].float()                          # [T][G][d]
        codes, scales = pool[name].view(-1, x.shape[1], P // B, B, D), pool[name + "_scale"]
        most = torch.zeros((T, x.shape[1]), device="cuda").scatter_reduce(
            0, run[:, None].expand(T, x.shape[1]), x.abs().amax(-1), "amax")
        e = _exponent(most)                                    # [blocks][G]
        before = scales[old_page, :, old_block].int() - 127    # [S][G]
        e = e.scatter_reduce(0, first_run[:, None].expand_as(before), torch.where(some, before, E_LO).to(e.dtype), "amax")
        now = e[first_run]
        old = codes[old_page, :, old_block]                    # [S][G][32][d]
        again = _code(_value(old, before[..., None, None]), now[..., None, None])
        codes[old_page, :, old_block] = torch.where(held, again, old)
        pool[name][page, :, slot] = _code(x, e[run][..., None])
        scales[page, :, slot // B] = (e[run] + 127).to(torch.uint8)
    return st["k"], st["v"], st["k_scale"], st["v_scale"]


def _rows(st, name, table, n):
    """The first n rows of a sequence, fp32 [G][n][128]."""
    x, e = _bytes(st)[name], _bytes(st)[name + "_scale"]
    pages = table[:(n + x.shape[2] - 1) // x.shape[2]].long()
    y = x[pages].view(pages.shape[0], x.shape[1], -1, B, D)
    y = _value(y, e[pages].int()[..., None, None] - 127)       # [pages][G][blocks][32][128]
    return y.transpose(0, 1).reshape(x.shape[1], -1, D)[:, :n]


def _queries(st, at, m):
    """m tokens' rows for each KV head, fp32 [G][heads of it x m][128]."""
    G, H = HEADS[st["case"]["heads"]]
    return st["q"][at:at + m].float().reshape(m, G, H // G, D).permute(1, 2, 0, 3).reshape(G, -1, D)


def _hidden(m, n, Hg, causal, window):
    if not causal:
        return None
    key = torch.arange(n, device="cuda")[None, :]
    mine = torch.arange(n - m, n, device="cuda").repeat(Hg)[:, None]
    return (key > mine) | (mine - key >= window) if window else key > mine


def _attend(st, causal, window):
    case, q = st["case"], st["q"]
    G, H = HEADS[case["heads"]]
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], device="cuda")
    at = 0
    for s, (m, n) in enumerate(zip(*_lengths(case))):
        K, V = _rows(st, "k", st["table"][s], n), _rows(st, "v", st["table"][s], n)
        x = _queries(st, at, m)
        hide = _hidden(m, n, H // G, causal, window)
        y, z = torch.empty_like(x), torch.empty(x.shape[:2], device="cuda")
        step = max(1, (1 << 28) // (x.shape[1] * n))           # heads at a time: 1 GB of scores
        for g in range(0, G, step):
            p = torch.matmul(x[g:g + step], K[g:g + step].transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
            if hide is not None:
                p.masked_fill_(hide, -math.inf)
            most = p.amax(dim=-1, keepdim=True)
            p = torch.exp(p - most)
            total = p.sum(dim=-1, keepdim=True)
            y[g:g + step] = torch.matmul(p, V[g:g + step]) / total
            z[g:g + step] = (most + torch.log(total))[..., 0]
        out[at:at + m] = y.reshape(G, H // G, m, D).permute(2, 0, 1, 3).reshape(m, H, D).to(q.dtype)
        lse[at:at + m] = z.reshape(G, H // G, m).permute(2, 0, 1).reshape(m, H)
        at += m
    return out, lse


def _plain_attn(st):
    out, lse = _attend(st, st["case"]["causal"], st["case"]["window"])
    return (out, lse) if st["case"]["lse"] else out


def _plain_mass(st):
    """mass[s][g][t] += the weights that the new tokens' queries pay key t; new keys start from nothing."""
    case = st["case"]
    G, H = HEADS[case["heads"]]
    at = 0
    for s, (m, n) in enumerate(zip(*_lengths(case))):
        K, x = _rows(st, "k", st["table"][s], n), _queries(st, at, m)
        z = st["lse"][at:at + m].reshape(m, G, H // G).permute(1, 2, 0).reshape(G, -1, 1)
        hide = _hidden(m, n, H // G, True, 0)
        st["out"][s, :, :n - m] = st["mass"][s, :, :n - m]
        st["out"][s, :, n - m:n] = 0
        step = max(1, (1 << 28) // (x.shape[1] * n))
        for g in range(0, G, step):
            p = torch.matmul(x[g:g + step], K[g:g + step].transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
            p = torch.exp(p - z[g:g + step]).masked_fill_(hide, 0.0)
            st["out"][s, g:g + step, :n] += p.sum(dim=1)
        at += m
    return st["out"]


def _plain_evict(st):
    case, pool = st["case"], _bytes(st)
    P, keep = case["page"], case["keep"]
    n = st["kv_len"].long()[:, None, None]
    S, G, L = st["mass"].shape
    t = torch.arange(L, device="cuda")
    m = n.clamp(max=keep)
    rank = torch.where(t < n, st["mass"], -1.0)
    rank = torch.where((t < n) & ((t < case["first"]) | (t >= n - case["recent"])), math.inf, rank)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    i = torch.arange(keep, device="cuda")
    index = torch.sort(torch.where(i < m, order, L), dim=-1).values
    stay = index < L                                           # [S][G][keep]
    index = torch.where(stay, index, 0)
    seq, head = torch.arange(S, device="cuda")[:, None, None], torch.arange(G, device="cuda")[:, None]
    page, slot = st["table"][seq, index // P].long(), index % P
    to, at = st["into"][torch.arange(S, device="cuda")[:, None], i // P].long()[:, None, :], i % P
    pad = -keep % B
    for name in ("k", "v"):
        e = pool[name + "_scale"][page, head, slot // B].int() - 127
        x = torch.where(stay[..., None], _value(pool[name][page, head, slot], e[..., None]), 0.0)
        x = torch.nn.functional.pad(x, (0, 0, 0, pad)).view(S, G, -1, B, D)
        e = _exponent(x.abs().amax(dim=(-2, -1)))              # [S][G][blocks]
        codes = _code(x, e[..., None, None]).view(S, G, -1, D)[:, :, :keep]
        pool[name][to, head, at] = torch.where(stay[..., None], codes, pool[name][to, head, at])
        first = slice(0, keep, B)
        scales = pool[name + "_scale"]
        scales[to[..., first], head, at[first] // B] = torch.where(
            stay[..., first], (e + 127).to(torch.uint8), scales[to[..., first], head, at[first] // B])
    mass = torch.where(stay, st["mass"].gather(2, index), 0.0)
    return (torch.where(stay, index, -1).to(torch.int32), mass, m[:, 0, 0].to(torch.int32),
            st["k"], st["v"], st["k_scale"], st["v_scale"])


def _plain_gather(st):
    n, dt = st["case"]["n"], _dt(st["case"])
    return tuple(_rows(st, x, st["table"][0], n).transpose(0, 1).to(dt).contiguous() for x in ("k", "v"))


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"append": _plain_append, "attn": _plain_attn, "mass": _plain_mass, "evict": _plain_evict,
                "gather": _plain_gather}[op](st)
    import paper_2607_15498_amd as vr
    if op == "append":
        vr.paged8_append(st["pages"], st["batch"], st["k_new"], st["v_new"])
        return st["pages"].k, st["pages"].v, st["pages"].k_scale, st["pages"].v_scale
    if op == "attn":
        lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda") if case["lse"] else None
        out = vr.paged8_attn(st["pages"], st["batch"], st["q"], causal=case["causal"], window=case["window"], lse=lse)
        return (out, lse) if case["lse"] else out
    if op == "mass":
        return vr.paged8_mass(st["pages"], st["batch"], st["q"], st["lse"], st["mass"], out=st["out"])
    if op == "evict":
        index, mass, kv_len = vr.paged8_evict(st["pages"], st["table"], st["kv_len"], st["mass"], case["keep"], st["into"],
                                              first=case["first"], recent=case["recent"])
        return index, mass, kv_len, st["pages"].k, st["pages"].v, st["pages"].k_scale, st["pages"].v_scale
    return vr.paged8_gather(st["pages"], st["table"][0], case["n"], dtype=_dt(case))


# ---- what a pass cannot do without, and its results in 64 bits -------------------------------

def _pairs(case):
    """Visible (query token, key) pairs of the batch."""
    total, causal, window = 0, case.get("causal", True), case.get("window", 0)
    for m, n in zip(*_lengths(case)):
        if not causal:
            total += m * n
            continue
        for p in range(n - m, n):
            total += min(p + 1, window) if window else p + 1
    return total


def work(case):
    G, H = HEADS[case["heads"]]
    row = D + 1.0 / B                                          # a row's codes and its part of a scale
    if case["op"] == "evict":
        kv_len = [int(n) for n in case["kv_len"].split(",")]
        stay = sum(min(n, case["keep"]) for n in kv_len)
        return {"bytes": G * (4 * sum(kv_len) + stay * (4 * row + 8)), "flops": 0}
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "gather":
        return {"bytes": 2 * case["n"] * G * (row + D * es), "flops": 0}
    q_len, kv_len = _lengths(case)
    T = sum(q_len)
    if case["op"] == "append":
        return {"bytes": 2 * T * G * (row + D * es), "flops": 0}
    if case["op"] == "mass":
        return {"bytes": sum(kv_len) * G * (row + 8) + T * H * (D * es + 4), "flops": 2 * D * H * _pairs(case)}
    # keys that no query of the sequence sees (behind the window) are not read
    seen = [min(n, m - 1 + case["window"]) if case["window"] else n for m, n in zip(q_len, kv_len)]
    return {"bytes": 2 * sum(seen) * G * row + 2 * T * H * D * es + (4 * T * H if case["lse"] else 0),
            "flops": 4 * D * H * _pairs(case)}


def _scale_of(amax):
    """The smallest power of two that takes amax (64 bits) to 448 or less, within the scales there are."""
    s = torch.full_like(amax, 2.0 ** E_LO)
    while bool((more := (amax > 448.0 * s) & (s < 2.0 ** E_HI)).any()):
        s = torch.where(more, 2.0 * s, s)
    return s


def _nearest(x):
    """x (64 bits) rounded to the nearest e4m3 value, ties to even codes."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _held(st, name):
    """Codes and scales of the pool as the numbers they are, 64 bits: [pages][G][blocks][32][d], [pages][G][blocks]."""
    x, s = st[name].to(torch.float32).to(torch.float64), st[name + "_scale"].view(torch.uint8).to(torch.float64)
    return x.reshape(x.shape[0], x.shape[1], -1, B, D), torch.exp2(s - 127.0)


def _sequence(st, name, pages, n):
    """A sequence's first n rows, 64 bits [G][n][d]."""
    x, s = st[name], st[name + "_scale"].view(torch.uint8)
    P = x.shape[2]
    pages = pages[:(n + P - 1) // P]
    y = torch.cat([x[i].to(torch.float64) * torch.exp2(s[i].to(torch.float64) - 127.0).repeat_interleave(B, dim=1)[..., None]
                   for i in pages], dim=1)
    return y[:, :n]


def exact(case, seed):
    st = prepare(case, seed)
    G, H = HEADS[case["heads"]]
    P, op = case["page"], case["op"]
    table = st["table"].tolist()
    if op == "gather":
        return tuple(_sequence(st, x, table[0], case["n"]).swapaxes(0, 1) for x in ("k", "v"))
    if op == "append":
        both, scales = [], []
        for name in ("k", "v"):
            x, s = _held(st, name)
            at = 0
            for q, (m, n) in enumerate(zip(*_lengths(case))):
                a = n - m
                while a < n:                                   # the part of the chunk in one block
                    b = min(n, (a // B + 1) * B)
                    page, block = table[q][a // P], a % P // B
                    new = st[name + "_new"][at:at + b - a].to(torch.float64).swapaxes(0, 1)     # [G][rows][d]
                    now = _scale_of(new.abs().amax(dim=(1, 2)))
                    if a % B:
                        was = s[page, :, block]
                        now = torch.maximum(now, was)
                        x[page, :, block, :a % B] = _nearest(x[page, :, block, :a % B] * (was / now)[:, None, None])
                    x[page, :, block, a % B:a % B + b - a] = _nearest(new / now[:, None, None])
                    s[page, :, block] = now
                    at, a = at + b - a, b
            both.append(x.reshape(st[name].shape))
            scales.append(s)
        return both[0], both[1], scales[0], scales[1]
    if op == "evict":
        keep, kv_len, L = case["keep"], st["kv_len"].tolist(), st["mass"].shape[2]
        index = torch.full((len(kv_len), G, keep), -1, dtype=torch.int32, device="cuda")
        mass = torch.zeros((len(kv_len), G, keep), dtype=torch.float64, device="cuda")
        into, held = st["into"].tolist(), {n: _held(st, n) for n in ("k", "v")}
        for q, n in enumerate(kv_len):
            m = min(n, keep)
            rows = {x: _sequence(st, x, table[q], n) for x in ("k", "v")}
            for g in range(G):
                w = st["mass"][q, g, :n].to(torch.float64)
                w[:case["first"]] = w[n - min(n, case["recent"]):] = math.inf
                # the m-th largest, and of those equal to it the first
                least = w.sort(descending=True).values[m - 1]
                mine = w > least
                equal = (w == least).nonzero()[:, 0]
                mine[equal[:m - int(mine.sum())]] = True
                index[q, g, :m] = chosen = mine.nonzero()[:, 0].to(torch.int32)
                mass[q, g, :m] = st["mass"][q, g][chosen].to(torch.float64)
                for x in ("k", "v"):
                    y = rows[x][g, chosen]
                    full = torch.zeros((-(-m // B), B, D), dtype=torch.float64, device="cuda")
                    full.view(-1, D)[:m] = y
                    s = _scale_of(full.abs().amax(dim=(1, 2)))
                    full = _nearest(full / s[:, None, None])
                    for i in range(full.shape[0]):
                        page, block = into[q][i * B // P], i * B % P // B
                        r = min(B, m - i * B)
                        held[x][0][page, g, block, :r] = full[i, :r]
                        held[x][1][page, g, block] = s[i]
        return (index, mass, torch.tensor([min(n, keep) for n in kv_len], dtype=torch.int32, device="cuda"),
                held["k"][0].reshape(st["k"].shape), held["v"][0].reshape(st["v"].shape), held["k"][1], held["v"][1])
    total = st["mass"].to(torch.float64) if op == "mass" else None
    if op == "mass":
        total[:] = 0
    out = torch.empty((st["q"].shape[0], H, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((st["q"].shape[0], H), dtype=torch.float64, device="cuda")
    at = 0
    for s, (m, n) in enumerate(zip(*_lengths(case))):
        K, V = (_sequence(st, x, table[s], n) for x in ("k", "v"))
        if op == "mass":
            total[s, :, :n - m] = st["mass"][s, :, :n - m].to(torch.float64)
        for h in range(H):
            g = h // (H // G)
            for a in range(0, m, 1024):
                b = min(m, a + 1024)
                w = (st["q"][at + a:at + b, h].to(torch.float64) @ K[g].T) / math.sqrt(D)
                if case.get("causal", True):
                    far = torch.arange(n - m + a, n - m + b, device="cuda")[:, None] - torch.arange(n, device="cuda")[None, :]
                    seen = far >= 0
                    if case.get("window", 0):
                        seen &= far < case["window"]
                    w = torch.where(seen, w, -math.inf)
                if op == "mass":
                    total[s, g, :n] += torch.exp(w - st["lse"][at + a:at + b, h].to(torch.float64)[:, None]).sum(dim=0)
                else:
                    lse[at + a:at + b, h] = torch.logsumexp(w, dim=-1)
                    out[at + a:at + b, h] = torch.softmax(w, dim=-1) @ V[g]
        at += m
    return total if op == "mass" else (out, lse) if case["lse"] else out
