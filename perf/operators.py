"""Serving a sequence before it is compressed: norm and rotate the queries and keys of new tokens, append
their rows to a paged cache, attend over that cache, and gather a sequence's rows for the codec.

Each case is one call of one operator.  Where `own` is false the operators are computed from elementary
torch operations in 32 bits, rounded once at the end; where it is true, by the package's entry points.
Head geometries are those of the repository's workloads: Llama (8 KV heads, 32 query heads), Qwen (4 and
28) and the tiny one (1 and 2), head dimension 128.
"""
import math

import torch

own = False

D = 128
HEADS = {"tiny": (1, 2), "qwen": (4, 28), "llama": (8, 32)}
EPS = 1e-6


def _norm(heads, T, *, dtype="bf16", norm="shared", rotate=True, fused=True, first=0):
    """norm: "none", "shared" (one weight for all heads) or "each" (one per head); fused: the rows are
    slices of one projection [T][(H + 2 G) d]; first: the position of the first token."""
    return {"op": "norm_rotate", "heads": heads, "T": T, "dtype": dtype, "norm": norm, "rotate": rotate,
            "fused": fused, "first": first}


def _text(lengths):
    return ",".join(str(n) for n in lengths)


def _lengths(case):
    """(new tokens, cached tokens with them) of every sequence."""
    return tuple([int(n) for n in case[k].split(",")] for k in ("q_len", "kv_len"))


def _append(heads, q_len, kv_len, *, page=64, dtype="bf16", rotate=True):
    return {"op": "append", "heads": heads, "q_len": _text(q_len), "kv_len": _text(kv_len), "page": page,
            "dtype": dtype, "rotate": rotate}


def _attn(heads, q_len, kv_len, *, page=64, dtype="bf16", causal=True, window=0):
    """q_len[s] new tokens of sequence s at the end of its kv_len[s] cached ones."""
    return {"op": "attn", "heads": heads, "q_len": _text(q_len), "kv_len": _text(kv_len), "page": page,
            "dtype": dtype, "causal": causal, "window": window}


def _gather(heads, n, *, page=64, dtype="bf16"):
    return {"op": "gather", "heads": heads, "n": n, "page": page, "dtype": dtype}


def listed():
    cases = {
        # one decode step of one sequence: latency is all it costs
        "norm_rotate_step": _norm("llama", 1, first=32767),
        # a whole Qwen-shaped prompt, rows sliced from the fused projection
        "norm_rotate_qwen_16k": _norm("qwen", 16384),
        # one decode step of 64 sequences of unlike lengths
        "append_step_b64": _append("llama", [1] * 64, [17 + 509 * s for s in range(64)], page=16),
        # a whole prompt written at once
        "append_llama_32k": _append("llama", [32768], [32768]),
        # the smallest attention: fp32, one KV head, 512 tokens
        "attn_step_tiny_f32": _attn("tiny", [1], [512], dtype="f32"),
        # one decode step of a long uncompressed sequence
        "attn_step_llama_32k": _attn("llama", [1], [32768]),
        # one decode step of a batch
        "attn_step_qwen_16k_b8": _attn("qwen", [1] * 8, [16384] * 8),
        # chunked prefill: the last 2048 tokens of a 32768-token prompt
        "attn_chunk_llama_32k": _attn("llama", [2048], [32768]),
        # a serving step: one odd chunk beside 16 sequences that decode
        "attn_mixed_b17": _attn("llama", [1003] + [1] * 16, [5003] + [301 + 523 * s for s in range(16)], page=16),
        # two odd prompts of an fp32 layer, from their first token
        "attn_prompts_f32": _attn("llama", [1531, 777], [1531, 777], dtype="f32", page=32),
        # a short fp32 sequence of odd length handed to the codec
        "gather_777_f32": _gather("llama", 777, page=16, dtype="f32"),
        # the headline prompt handed to the codec
        "gather_llama_32k": _gather("llama", 32768),
    }
    return [dict(c, name=k) for k, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rotate", "append", "attn", "attn", "attn", "gather"])
    heads = rng.choice(["llama", "llama", "qwen", "qwen", "tiny"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "norm_rotate":
        norm = rng.choice(["none", "shared", "shared", "each"])
        return _norm(heads, _log(rng, 1, 6000 if dtype == "f32" else 12000), dtype=dtype, norm=norm,
                     rotate=norm == "none" or rng.random() < 0.8, fused=rng.random() < 0.6,
                     first=rng.choice([0, _log(rng, 1, 1 << 20)]))
    if op == "gather":
        return _gather(heads, _log(rng, 1, 16384 if dtype == "f32" else 32768), page=page, dtype=dtype)
    if op == "append":
        S = rng.choice([1, 1, 3, 16, 64])
        q_len = [_log(rng, 1, 16384 // S) if rng.random() < 0.5 else 1 for _ in range(S)]
        kv_len = [q + rng.choice([0, _log(rng, 1, 16384 // S)]) for q in q_len]
        return _append(heads, q_len, kv_len, page=page, dtype=dtype, rotate=rng.random() < 0.7)
    kind = rng.choice(["step", "step", "chunk", "prompt", "mixed"])
    window = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
    causal = True
    if kind == "step":
        S = rng.choice([1, 1, 4, 16])
        kv_len = [_log(rng, 1, (32768 if dtype == "f32" else 65536) // S) for _ in range(S)]
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
    return _attn(heads, q_len, kv_len, page=page, dtype=dtype, causal=causal, window=window if causal else 0)


# ---- inputs ------------------------------------------------------------------------------

def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _theta():
    """Llama-3.1's per-pair rotary frequencies (base 500000, long-context scaling 8), fp32."""
    inv = 500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    smooth = ((8192.0 / (2.0 * math.pi / inv) - 1.0) / 3.0).clamp(0.0, 1.0)
    return ((1.0 - smooth) * inv / 8.0 + smooth * inv).float().cuda()


def _keys(gen, shape, u):
    """Keys whose channels decay, two outlier channels, 5% of the tokens planted along u."""
    sk = (1.0 / torch.arange(1, D + 1, dtype=torch.float32, device="cuda")).sqrt()
    sk[1:3] = 4.0
    k = torch.randn(shape, generator=gen, device="cuda") * sk
    hit = torch.rand(shape[:-1], generator=gen, device="cuda")
    return k + torch.where(hit < 0.05, 4.0 + 40.0 * hit, 0.0)[..., None] * u


def _pool(case, gen, dt, kv_len, u, filled):
    """A pool of pages in shuffled order, some of them nobody's, and the sequences' page table."""
    G, _ = HEADS[case["heads"]]
    P = case["page"]
    need = [(n + P - 1) // P for n in kv_len]
    total = sum(need) + 3
    shape = (total, G, P, D)
    if filled:
        k = _keys(gen, shape, u[:, None, :]).to(dt)
        v = torch.randn(shape, generator=gen, device="cuda").to(dt)
    else:
        k, v = torch.zeros(shape, dtype=dt, device="cuda"), torch.zeros(shape, dtype=dt, device="cuda")
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(kv_len), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    return k, v, table


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    G, H = HEADS[case["heads"]]
    dt = _dt(case)
    st = {"case": case}
    u = torch.randn((G, D), generator=gen, device="cuda")
    u = u / u.norm(dim=1, keepdim=True)
    if case["op"] == "norm_rotate":
        T = case["T"]
        if case["fused"]:
            x = torch.randn((T, H + 2 * G, D), generator=gen, device="cuda").to(dt)
            st["q"], st["k"] = x[:, :H], x[:, H:H + G]
        else:
            st["q"] = torch.randn((T, H, D), generator=gen, device="cuda").to(dt)
            st["k"] = _keys(gen, (T, G, D), u).to(dt)
        st["pos"] = torch.arange(case["first"], case["first"] + T, dtype=torch.int32, device="cuda")
        st["theta"] = _theta() if case["rotate"] else None
        st["wq"] = st["wk"] = None
        if case["norm"] != "none":
            each = case["norm"] == "each"
            st["wq"] = 1.0 + 0.2 * torch.randn((H, D) if each else (D,), generator=gen, device="cuda")
            st["wk"] = 1.0 + 0.2 * torch.randn((G, D) if each else (D,), generator=gen, device="cuda")
        return st
    if case["op"] == "gather":
        st["k"], st["v"], st["table"] = _pool(case, gen, dt, [case["n"]], u, True)
    else:
        q_len, kv_len = _lengths(case)
        T = sum(q_len)
        st["k"], st["v"], st["table"] = _pool(case, gen, dt, kv_len, u, case["op"] == "attn")
        st["kv_len"] = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
        st["q_start"] = torch.tensor([sum(q_len[:s]) for s in range(len(q_len) + 1)], dtype=torch.int32, device="cuda")
        if case["op"] == "append":
            st["k_new"] = _keys(gen, (T, G, D), u).to(dt)
            st["v_new"] = torch.randn((T, G, D), generator=gen, device="cuda").to(dt)
            st["theta"] = _theta() if case["rotate"] else None
        else:
            heads = torch.arange(H, device="cuda") // (H // G)
            q = math.sqrt(D) * u[heads] + 0.5 * torch.randn((T, H, D), generator=gen, device="cuda")
            st["q"] = q.to(dt)
    if own:
        import paper_2607_15498_amd as vr
        st["pages"] = vr.PagedCache(st["k"], st["v"])
        if case["op"] != "gather":
            st["batch"] = vr.PagedBatch(st["table"], st["kv_len"], st["q_start"])
    return st


# ---- the operators -------------------------------------------------------------------------

def _turn(x, pos, theta):
    """x [T][heads][128] (fp32) turned at positions pos; the angles in 64 bits, as far positions need."""
    a = pos.double()[:, None] * theta.double()[None, :]
    c, s = a.cos().float()[:, None, :], a.sin().float()[:, None, :]
    x0, x1 = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([x0 * c - x1 * s, x0 * s + x1 * c], dim=-1)


def _plain_norm_rotate(st):
    out = []
    for x, w in ((st["q"], st["wq"]), (st["k"], st["wk"])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + EPS) * w
        if st["theta"] is not None:
            y = _turn(y, st["pos"], st["theta"])
        out.append(y.to(x.dtype))
    return tuple(out)


def _plain_append(st):
    P, start = st["case"]["page"], st["q_start"].long()
    i = torch.arange(st["k_new"].shape[0], device="cuda")
    s = torch.searchsorted(start[1:], i, right=True)           # the token's sequence
    t = st["kv_len"].long()[s] - start[s + 1] + i              # and its position there
    page, slot = st["table"][s, t // P].long(), t % P
    k = st["k_new"]
    if st["theta"] is not None:
        k = _turn(k.float(), t, st["theta"]).to(k.dtype)
    st["k"][page, :, slot] = k
    st["v"][page, :, slot] = st["v_new"]
    return st["k"], st["v"]


def _rows(x, table, n):
    """The first n rows of a sequence, fp32 [G][n][128]."""
    P = x.shape[2]
    y = x[table[:(n + P - 1) // P].long()]                     # [pages][G][P][128]
    return y.transpose(0, 1).reshape(x.shape[1], -1, D)[:, :n].float()


def _plain_attn(st):
    case, q = st["case"], st["q"]
    G, H = HEADS[case["heads"]]
    out = torch.empty_like(q)
    at = 0
    for s, (m, n) in enumerate(zip(*_lengths(case))):
        K, V = _rows(st["k"], st["table"][s], n), _rows(st["v"], st["table"][s], n)
        x = q[at:at + m].float().reshape(m, G, H // G, D).permute(1, 2, 0, 3).reshape(G, -1, D)
        key = torch.arange(n, device="cuda")[None, :]
        mine = torch.arange(n - m, n, device="cuda").repeat(H // G)[:, None]
        hide = None
        if case["causal"]:
            hide = key > mine
            if case["window"]:
                hide = hide | (mine - key >= case["window"])
        y = torch.empty_like(x)
        step = max(1, (1 << 28) // (x.shape[1] * n))           # heads at a time: 1 GB of scores
        for g in range(0, G, step):
            p = torch.matmul(x[g:g + step], K[g:g + step].transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
            if hide is not None:
                p.masked_fill_(hide, -math.inf)
            p = torch.exp(p - p.amax(dim=-1, keepdim=True))
            y[g:g + step] = torch.matmul(p, V[g:g + step]) / p.sum(dim=-1, keepdim=True)
        out[at:at + m] = y.reshape(G, H // G, m, D).permute(2, 0, 1, 3).reshape(m, H, D).to(q.dtype)
        at += m
    return out


def _plain_gather(st):
    n = st["case"]["n"]
    dt = st["k"].dtype
    return tuple(_rows(x, st["table"][0], n).transpose(0, 1).contiguous().to(dt) for x in (st["k"], st["v"]))


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"norm_rotate": _plain_norm_rotate, "append": _plain_append, "attn": _plain_attn,
                "gather": _plain_gather}[op](st)
    import paper_2607_15498_amd as vr
    if op == "norm_rotate":
        return vr.norm_rotate(st["q"], st["k"], pos=st["pos"], theta=st["theta"], wq=st["wq"], wk=st["wk"], eps=EPS)
    if op == "append":
        vr.paged_append(st["pages"], st["batch"], st["k_new"], st["v_new"], theta=st["theta"])
        return st["pages"].k, st["pages"].v
    if op == "attn":
        return vr.paged_attn(st["pages"], st["batch"], st["q"], causal=st["case"]["causal"], window=st["case"]["window"])
    return vr.paged_gather(st["pages"], st["table"][0], st["case"]["n"])


# ---- what a pass cannot do without, and its results in 64 bits -------------------------------

def _pairs(case):
    """Visible (query token, key) pairs of the batch."""
    total = 0
    for m, n in zip(*_lengths(case)):
        if not case["causal"]:
            total += m * n
            continue
        for p in range(n - m, n):
            total += min(p + 1, case["window"]) if case["window"] else p + 1
    return total


def work(case):
    G, H = HEADS[case["heads"]]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm_rotate":
        n = case["T"] * (H + G) * D
        per = (4 if case["norm"] != "none" else 0) + (3 if case["rotate"] else 0)
        return {"bytes": 2 * n * es + 4 * case["T"], "flops": per * n}
    if case["op"] == "gather":
        return {"bytes": 4 * case["n"] * G * D * es, "flops": 0}
    T = sum(_lengths(case)[0])
    if case["op"] == "append":
        return {"bytes": 4 * T * G * D * es, "flops": (3 if case["rotate"] else 0) * T * G * D}
    # keys that no query of the sequence sees (behind the window) are not read
    seen = [min(n, m - 1 + case["window"]) if case["window"] else n for m, n in zip(*_lengths(case))]
    return {"bytes": (2 * sum(seen) * G + 2 * T * H) * D * es, "flops": 4 * D * H * _pairs(case)}


def exact(case, seed):
    st = prepare(case, seed)
    G, H = HEADS[case["heads"]]
    if case["op"] == "norm_rotate":
        both = []
        for x, w in ((st["q"], st["wq"]), (st["k"], st["wk"])):
            z = x.to(torch.float64)
            if w is not None:
                z = z / (z.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.to(torch.float64)
            if st["theta"] is not None:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                                   torch.outer(st["pos"].to(torch.float64), st["theta"].to(torch.float64)))[:, None]
                z = torch.complex(z[..., :64].contiguous(), z[..., 64:].contiguous()) * turn
                z = torch.cat([z.real, z.imag], dim=-1)
            both.append(z)
        return tuple(both)
    if case["op"] == "gather":
        P, n = case["page"], case["n"]
        page = st["table"][0].tolist()
        both = []
        for x in (st["k"], st["v"]):
            y = torch.empty((n, G, D), dtype=torch.float64, device="cuda")
            for i in range((n + P - 1) // P):
                m = min(P, n - i * P)
                y[i * P:i * P + m] = x[page[i], :, :m].swapaxes(0, 1)
            both.append(y)
        return tuple(both)
    P, table = case["page"], st["table"].tolist()
    at = 0
    if case["op"] == "append":
        k, v = st["k"].to(torch.float64), st["v"].to(torch.float64)
        for s, (m, n) in enumerate(zip(*_lengths(case))):
            t = torch.arange(n - m, n, device="cuda", dtype=torch.float64)
            z = st["k_new"][at:at + m].to(torch.float64)
            if st["theta"] is not None:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(t, st["theta"].to(torch.float64)))
                z = torch.complex(z[..., :64].contiguous(), z[..., 64:].contiguous()) * turn[:, None]
                z = torch.cat([z.real, z.imag], dim=-1)
            a = n - m
            while a < n:                                       # the part of the chunk on one page
                b = min(n, (a // P + 1) * P)
                i = a - (n - m)
                k[table[s][a // P], :, a % P:a % P + b - a] = z[i:i + b - a].swapaxes(0, 1)
                v[table[s][a // P], :, a % P:a % P + b - a] = st["v_new"][at + i:at + i + b - a].to(torch.float64).swapaxes(0, 1)
                a = b
            at += m
        return k, v
    out = torch.empty((st["q"].shape[0], H, D), dtype=torch.float64, device="cuda")
    for s, (m, n) in enumerate(zip(*_lengths(case))):
        pages = [table[s][i] for i in range((n + P - 1) // P)]
        for g in range(G):
            K = torch.cat([st["k"][i, g] for i in pages])[:n].to(torch.float64)
            V = torch.cat([st["v"][i, g] for i in pages])[:n].to(torch.float64)
            for h in range(g * (H // G), (g + 1) * (H // G)):
                for a in range(0, m, 1024):
                    b = min(m, a + 1024)
                    w = (st["q"][at + a:at + b, h].to(torch.float64) @ K.T) / math.sqrt(D)
                    if case["causal"]:
                        far = torch.arange(n - m + a, n - m + b, device="cuda")[:, None] - torch.arange(n, device="cuda")[None, :]
                        seen = far >= 0
                        if case["window"]:
                            seen &= far < case["window"]
                        w = torch.where(seen, w, -math.inf)
                    out[at + a:at + b, h] = torch.softmax(w, dim=-1) @ V
        at += m
    return out
