"""Paged cache, without a GPU: the C ABI's refusals, the structs' layout, the index arithmetic that the kernels
share with the host (walked in a host build: every new token meets every key that it sees exactly once, whatever the
device arrays hold), and the generated code of the attention kernel, whose accumulators are registers named in inline
assembly."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED = 0, -1, -3


@pytest.fixture(scope="module")
def L():
    from paper_2607_15498_amd import _lib
    return _lib.load()


def test_struct_layouts_match_header(tmp_path):
    from paper_2607_15498_amd import _lib
    want, lines = [], []
    for c, py in (("varrate_pages", _lib.PagesC), ("varrate_batch", _lib.BatchC)):
        lines.append(f'printf("%zu\\n", sizeof({c}));')
        want.append(ctypes.sizeof(py))
        for name, _ in py._fields_:
            lines.append(f'printf("%zu\\n", offsetof({c}, {name}));')
            want.append(getattr(py, name).offset)
    prog = tmp_path / "probe.c"
    prog.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "varrate.h"\nint main(void) {' + "".join(lines) + "return 0; }")
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(prog)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, check=True).stdout.split()]
    assert got == want


# ---- refusals: addresses are never followed, so any aligned number serves --------------------------------------------

A = 1 << 20


def pages(**kw):
    from paper_2607_15498_amd import _lib
    f = dict(k=A, v=2 * A, n_pages=8, G=2, d=128, page=64, dtype=_lib.VARRATE_BF16)
    f.update(kw)
    return _lib.PagesC(*(f[n] for n, _ in _lib.PagesC._fields_))


def batch(**kw):
    from paper_2607_15498_amd import _lib
    f = dict(table=3 * A, kv_len=4 * A, q_start=5 * A, table_stride=4, T=5, S=2, width=4)
    f.update(kw)
    return _lib.BatchC(*(f[n] for n, _ in _lib.BatchC._fields_))


def attn(L, pg=None, b=None, **kw):
    f = dict(q=6 * A, q_stride=4 * 128, H=4, causal=1, window=0, scale=0.1, out=7 * A, out_stride=4 * 128, ws=8 * A,
             ws_bytes=1 << 40)
    f.update(kw)
    return L.varrate_paged_attn(pg or pages(), b or batch(), f["q"], f["q_stride"], f["H"], f["causal"], f["window"],
                                f["scale"], f["out"], f["out_stride"], f["ws"], f["ws_bytes"], None)


def append(L, pg=None, b=None, **kw):
    f = dict(k=6 * A, ks=256, v=7 * A, vs=256, theta=None)
    f.update(kw)
    return L.varrate_paged_append(pg or pages(), b or batch(), f["k"], f["ks"], f["v"], f["vs"], f["theta"], None)


def gather(L, pg=None, **kw):
    f = dict(table=3 * A, width=4, n=100, K=6 * A, V=7 * A)
    f.update(kw)
    return L.varrate_paged_gather(pg or pages(), f["table"], f["width"], f["n"], f["K"], f["V"], None)


def norm(L, **kw):
    f = dict(dtype=1, T=3, q=A, qs=512, H=4, k=2 * A, ks=256, G=2, pos=3 * A, theta=4 * A, wq=5 * A, wqs=0, wk=6 * A,
             wks=128, eps=1e-6, qo=7 * A, qos=512, ko=8 * A, kos=256)
    f.update(kw)
    return L.varrate_norm_rotate(*f.values(), None)


BAD_PAGES = [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=A + 8), EINVAL), (dict(v=A + 2), EINVAL),
    (dict(n_pages=0), EINVAL), (dict(n_pages=1 << 31), EINVAL), (dict(n_pages=-1), EINVAL), (dict(G=0), EINVAL),
    (dict(G=1025), EINVAL), (dict(d=64), EUNSUPPORTED), (dict(d=0), EUNSUPPORTED), (dict(page=8), EUNSUPPORTED),
    (dict(page=48), EUNSUPPORTED), (dict(page=512), EUNSUPPORTED), (dict(page=0), EUNSUPPORTED),
    (dict(page=-64), EUNSUPPORTED), (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL),
]
BAD_BATCHES = [
    (dict(table=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(q_start=None), EINVAL), (dict(table=A + 2), EINVAL),
    (dict(kv_len=A + 1), EINVAL), (dict(q_start=A + 3), EINVAL), (dict(S=0), EINVAL), (dict(S=-1), EINVAL),
    (dict(S=65537), EINVAL), (dict(T=-1), EINVAL), (dict(width=0), EINVAL), (dict(width=-4), EINVAL),
    (dict(width=(1 << 24) + 1), EINVAL), (dict(width=(1 << 31) - 1), EINVAL), (dict(table_stride=-1), EINVAL),
    (dict(T=1 << 30), EUNSUPPORTED), (dict(T=(1 << 63) - 1), EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_pages_refused(L, kw, code):
    p = pages(**kw)
    for call in (attn, append, gather):
        assert call(L, p) == code and L.varrate_last_error(), call.__name__
    assert L.varrate_paged_attn_workspace_bytes(p, batch(), 4) == 0


@pytest.mark.parametrize("kw,code", BAD_BATCHES)
def test_batches_refused(L, kw, code):
    b = batch(**kw)
    for call in (attn, append):
        assert call(L, None, b) == code and L.varrate_last_error(), call.__name__
    assert L.varrate_paged_attn_workspace_bytes(pages(), b, 4) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q=A + 8), EINVAL), (dict(out=A + 8), EINVAL),
    (dict(q_stride=4), EINVAL), (dict(q_stride=-512), EINVAL), (dict(out_stride=504), EINVAL), (dict(out_stride=0), EINVAL),
    (dict(out_stride=256), EINVAL), (dict(H=0), EINVAL), (dict(H=-2), EINVAL), (dict(H=3), EUNSUPPORTED),
    (dict(causal=2), EINVAL), (dict(causal=-1), EINVAL), (dict(window=-1), EINVAL), (dict(window=(1 << 30) + 1), EINVAL),
    (dict(causal=0, window=5), EUNSUPPORTED), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=1e38), EINVAL),
    (dict(scale=1e-38), EINVAL), (dict(out=6 * A), EINVAL), (dict(ws=None), EINVAL), (dict(ws_bytes=16), EINVAL),
    (dict(ws=A + 4), EINVAL),
])
def test_attn_refused(L, kw, code):
    assert attn(L, None, batch(width=8), **kw) == code and L.varrate_last_error()     # 512 keys: may be cut


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=A + 8), EINVAL), (dict(v=A + 8), EINVAL),
    (dict(ks=100), EINVAL), (dict(vs=-256), EINVAL), (dict(theta=A + 2), EINVAL),
])
def test_append_refused(L, kw, code):
    assert append(L, **kw) == code and L.varrate_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), EINVAL), (dict(table=A + 2), EINVAL), (dict(width=0), EINVAL), (dict(width=1 << 30), EINVAL),
    (dict(n=-1), EINVAL), (dict(n=257), EINVAL), (dict(n=1 << 40), EINVAL), (dict(K=None), EINVAL), (dict(V=None), EINVAL),
    (dict(K=A + 8), EINVAL), (dict(V=A + 8), EINVAL),
])
def test_gather_refused(L, kw, code):
    assert gather(L, **kw) == code and L.varrate_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), EINVAL), (dict(T=-1), EINVAL), (dict(H=0, G=0), EINVAL), (dict(H=-1), EINVAL), (dict(G=65537), EINVAL),
    (dict(T=1 << 28), EUNSUPPORTED), (dict(T=(1 << 63) - 1), EUNSUPPORTED), (dict(eps=-1e-6), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(pos=None), EINVAL), (dict(pos=A + 2), EINVAL),
    (dict(theta=A + 2), EINVAL), (dict(wq=A + 4), EINVAL), (dict(wqs=64), EINVAL), (dict(wks=-128), EINVAL),
    (dict(q=None), EINVAL), (dict(qo=None), EINVAL), (dict(k=None), EINVAL), (dict(ko=None), EINVAL), (dict(q=A + 8), EINVAL),
    (dict(ko=A + 8), EINVAL), (dict(qs=100), EINVAL), (dict(qos=128), EINVAL), (dict(kos=-256), EINVAL),
    (dict(qo=A, qos=1024), EINVAL), (dict(ko=2 * A, kos=512), EINVAL),
])
def test_norm_rotate_refused(L, kw, code):
    assert norm(L, **kw) == code and L.varrate_last_error()


def test_nothing_to_do(L):
    """No tokens: nothing is launched and no rows are needed."""
    b = batch(T=0)
    assert attn(L, None, b, q=None, out=None, ws=None, ws_bytes=0) == OK
    assert append(L, None, b, k=None, v=None) == OK
    assert gather(L, n=0, K=None, V=None) == OK
    assert norm(L, T=0, q=None, qo=None) == OK
    assert L.varrate_paged_attn_workspace_bytes(pages(), b, 4) == 0


def test_workspace_follows_the_table(L):
    """A table too short for a cut needs none; what a call may need grows with rows and table up to a bound."""
    need = lambda T, S, width, H=4, **kw: L.varrate_paged_attn_workspace_bytes(pages(**kw), batch(T=T, S=S, width=width), H)
    assert need(1, 1, 4) == 0 and need(1, 1, 2, dtype=0) == 0
    assert 0 < need(1, 1, 5) < need(1, 1, 64) < need(4, 4, 64) <= need(4, 4, 1 << 20)
    assert need(1 << 20, 1, 1 << 20) == need(1 << 22, 1, 1 << 20) == 1024 * 256 * 130 * 4 + 16


def test_binding_refuses_before_the_library(L):
    import torch
    import paper_2607_15498_amd as vr
    kv = torch.zeros((2, 1, 16, 128))
    with pytest.raises(vr.VarRateError):
        vr.PagedCache(kv, kv)                              # not on a device
    with pytest.raises(vr.VarRateError):
        vr.PagedCache(kv, kv[:1])
    with pytest.raises(vr.VarRateError):
        vr.PagedCache(kv[0], kv[0])
    with pytest.raises(vr.VarRateError):
        vr.PagedCache(kv.half(), kv.half())
    with pytest.raises(vr.VarRateError):
        vr.new_pages(2, 1, 16, dtype="fp16", device="cpu")
    i = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(vr.VarRateError):
        vr.PagedBatch(i, i[0, :1], i[0, :2])
    with pytest.raises(vr.VarRateError):
        vr.norm_rotate(torch.zeros((1, 2, 128)))
    with pytest.raises(vr.VarRateError):
        vr.norm_rotate(None)


# ---- the index arithmetic, in a host build ---------------------------------------------------------------------------

WALK = r'''
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <random>
#include <vector>
#include "vr_pages.h"
using namespace vr;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)
static std::mt19937 gen(7);
static int32_t pick_of(int32_t lo, int32_t hi) { return lo + (int32_t)(gen() % (uint32_t)(hi - lo + 1)); }

static void one_cut(const std::vector<SeqRange>& r, int32_t L, int G, int Hg, int causal, int window, Costs c, bool rising,
                    int64_t T, int64_t cap, bool taken) {
    int64_t pieces = 0, units = 0, recs = 0;
    for (SeqRange s : r) {
        const int64_t rows = seq_rows(s, Hg);
        const int bm = tile_rows(s, Hg), tiles = seq_tiles(s, Hg);
        CHECK((int64_t)tiles * bm >= rows && (int64_t)(tiles - 1) * bm < rows + (rows == 0));
        const int32_t span = seq_span(s, Hg, window), np = seq_pieces(span, key_cost(s, Hg, c), L, c.lmin);
        CHECK(np >= 1);
        pieces += (int64_t)tiles * np * G;
        units += (int64_t)tiles * G;
        if (np > 1) recs += (int64_t)tiles * np * G * bm;
        for (int tile = 0; tile < tiles; ++tile) {
            const int32_t row0 = tile * bm, n = (int32_t)std::min<int64_t>(bm, rows - row0);
            int32_t first = 0, last = 0, at = -1;
            for (int i = 0; i < n; ++i) {
                int32_t lo, hi;
                row_keys(s, (row0 + i) / Hg, causal, window, lo, hi);
                CHECK(lo >= 0 && hi >= 0 && hi <= s.klen);
                if (i == 0) first = lo;
                CHECK(lo >= first && hi >= last);           // both grow along the rows
                last = hi;
            }
            for (int p = 0; p < np; ++p) {
                int32_t lo, hi;
                piece_keys(s, row0, n, p, np, Hg, causal, window, lo, hi);
                if (hi <= lo) continue;
                CHECK(lo >= 0 && hi <= s.klen);
                if (at < 0) CHECK(lo == first);
                else CHECK(lo == at && lo % 64 == 0);       // pieces follow each other
                at = hi;
            }
            CHECK(at == last || (at < 0 && last <= first));
        }
    }
    if (taken && rising) {
        CHECK(units <= max_units(T, (int)r.size(), G, Hg));
        CHECK(pieces <= max_pieces(T, (int)r.size(), G, Hg, cap, c.lmin));
        CHECK(recs <= max_records(T, (int)r.size(), G, Hg, cap, c.lmin));
    }
}

int main() {
    const int heads[][2] = {{1, 1}, {8, 4}, {4, 7}, {1, 40}, {3, 1}, {2, 300}};
    for (int round = 0; round < 1500; ++round) {
        const int S = pick_of(1, round % 3 ? 5 : 40), T = pick_of(0, round % 5 == 0 ? 3000 : 130), cap = 16 * pick_of(1, round % 4 ? 300 : 12);
        const int* gh = heads[gen() % 6];
        const int G = gh[0], Hg = gh[1];
        const int causal = (int)(gen() % 4 != 0), window = causal && gen() % 2 ? pick_of(1, gen() % 2 ? 40 : 3000) : 0;
        const Costs c = costs_of(gen() % 2);
        std::vector<int32_t> start(S + 1), len(S);
        const bool rising = round % 4 != 3;
        for (int& x : start) x = pick_of(0, T);
        if (rising) std::sort(start.begin(), start.end());
        else for (int& x : start) if (gen() % 3 == 0) x = (int32_t)gen();
        for (int& x : len) x = gen() % 6 == 0 ? (int32_t)gen() : pick_of(0, cap);
        std::vector<SeqRange> r;
        Sums s;
        for (int i = 0; i < S; ++i) {
            r.push_back(seq_range(start[i], start[i + 1], len[i], T, cap));
            CHECK(r[i].q0 >= 0 && r[i].qlen >= 0 && r[i].q0 + r[i].qlen <= T && r[i].klen >= 0 && r[i].klen <= cap);
            sum_up(s, r[i], G, Hg, causal, window, c);
        }
        for (int t = 0; t < T; ++t) {
            const int q = find_seq(start.data(), S, t);
            if (q < 0) CHECK(t < start[0] || t >= start[S]);
            else CHECK(q < S && start[q] <= t && t < start[q + 1]);
            if (q >= 0) CHECK(t >= r[q].q0 && t < r[q].q0 + r[q].qlen);
        }
        float best = 0.f;
        Cut kept = {};
        for (int i = 0; i < CUTS; ++i) {
            Cut t = cut_begin(i, s.spans);
            CHECK(t.L >= 1);
            for (SeqRange x : r) cut_up(t, x, G, Hg, window, c);
            const float cost = cut_cost(t, s, c);
            CHECK(cost >= 0.f && cost <= 1e30f);
            if (i == 0 || cost < best) {
                best = cost;
                kept = t;
            }
            const bool taken = i == 0 || cost < 1e30f;
            int64_t pieces = 0;
            for (SeqRange x : r)
                pieces += (int64_t)seq_tiles(x, Hg) * G * seq_pieces(seq_span(x, Hg, window), key_cost(x, Hg, c), t.L, c.lmin);
            CHECK((float)pieces == t.pieces);
            one_cut(r, t.L, G, Hg, causal, window, c, rising, T, cap, taken && may_cut(s, c));
        }
        one_cut(r, pick_of(1, 5000), G, Hg, causal, window, c, rising, T, cap, false);
        if (rising) CHECK(s.units <= max_units(T, S, G, Hg));
    }
    // the longest: nothing overflows
    for (int bf = 0; bf < 2; ++bf) {
        const Costs c = costs_of(bf);
        const SeqRange r = seq_range(0, 1 << 20, 1 << 30, 1 << 20, 1 << 30);
        for (int32_t L : {1, 4096, 999999999, WHOLE}) {
            const int32_t np = seq_pieces(seq_span(r, 1024, 0), key_cost(r, 1024, c), L, c.lmin);
            CHECK(np >= 1 && (int64_t)np * piece_len(1 << 30, np) >= 1 << 30);
            int32_t lo, hi;
            piece_keys(r, (1 << 30) - 256, 256, np - 1, np, 1024, 1, 0, lo, hi);
            CHECK(lo <= hi && hi <= 1 << 30);
        }
    }
    // every piece of a call is one workgroup's, forwards and backwards
    for (uint32_t n : {8u, 16u, 248u, 256u})
        for (int rounds : {1, 2, 5}) {
            std::vector<int> hit(n * rounds, 0);
            for (uint32_t b = 0; b < n; ++b)
                for (int k = 0; k < rounds; ++k) {
                    const int64_t i = piece_number(b, n, b & 8 ? rounds - 1 - k : k);
                    CHECK(i >= 0 && i < (int64_t)hit.size() && i % 8 == b % 8);
                    ++hit[i];
                }
            for (int h : hit) CHECK(h == 1);
        }
    CHECK(good_page(-1, 5) == -1 && good_page(5, 5) == -1 && good_page(4, 5) == 4 && good_page(INT32_MIN, 5) == -1);
    printf("ok\n");
    return 0;
}
'''


def test_index_arithmetic(tmp_path):
    from paper_2607_15498_amd import build as B
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(WALK)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-Wall", "-I", B.CSRC,
                    str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-2000:]


# ---- the generated code of the bf16 attention ------------------------------------------------------------------------

OWN_AGPRS = 192                                            # a0 .. a191: sums and queries


def _registers(text):
    r = set()
    for kind, lo, hi in re.findall(r"\b([av])\[(\w+)(?::(\w+))?\]", text):
        r |= {kind + str(i) for i in range(int(lo, 0), int(hi or lo, 0) + 1)}
    return r | {k + n for k, n in re.findall(r"\b([av])(\d+)\b", text)}


class Instr:
    def __init__(self, text, asm):
        self.text, self.asm = text, asm
        self.op, _, rest = text.partition(" ")
        self.args = [x.strip() for x in re.split(r",(?![^\[]*\])", rest)]
        self.mfma = self.op.startswith("v_mfma")
        self.next = []
        writes = self.op.startswith(("v_", "ds_read", "global_load", "scratch_load")) and not self.op.startswith("v_cmp")
        self.dst = _registers(self.args[0]) if writes else set()
        self.src = _registers(",".join(self.args[1:] if writes else self.args))


def _instructions(body):
    """The kernel's instructions, each with those that may follow it."""
    out, labels, asm, jumps = [], {}, False, []
    for line in body.splitlines():
        if ";;#ASMSTART" in line:
            asm = True
        elif ";;#ASMEND" in line:
            asm = False
        code = line.split(";")[0].strip()
        m = re.match(r"^([.\w]+):", code)
        if m:
            labels[m.group(1)] = len(out)
        elif code and not code.startswith("."):
            out.append(Instr(code, asm))
    for i, x in enumerate(out):
        if x.op in ("s_branch",) or x.op.startswith("s_cbranch"):
            x.next.append(labels[x.args[0]])
        assert x.op not in ("s_setpc_b64", "s_swappc_b64"), "no calls"
        if x.op not in ("s_branch", "s_endpgm") and i + 1 < len(out):
            x.next.append(i + 1)
    return out


def _follow(code, start, states, visit):
    """visit(instruction, wait states since `start` was issued) along every path, until it returns True or `states` are
    over.  A product waits until the matrix cores are free of the one before: 8 states from its issue."""
    seen = set()
    work = [(n, 1, 8 if code[start].mfma else 0) for n in code[start].next]
    while work:
        i, t, free = work.pop()
        x = code[i]
        if x.mfma and t < free:
            t = free
        if t >= states or (i, t, free) in seen:
            continue
        seen.add((i, t, free))
        if visit(x, t):
            continue
        t2 = t + (int(x.args[0], 0) + 1 if x.op == "s_nop" else 1)
        work += [(n, t2, t + 8 if x.mfma else free) for n in x.next]


@pytest.fixture(scope="module")
def bf16_kernel(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    from paper_2607_15498_amd import build as B
    out = tmp_path_factory.mktemp("asm") / "paged_attn.s"
    cmd = ["hipcc", *B.FLAGS, *B.SOURCE_FLAGS["paged_attn.hip"], "-S", "--offload-device-only", os.path.join(B.CSRC, "paged_attn.hip"),
           "-o", str(out)]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    m = re.search(r"^(_ZN2vr17paged_attn_kernelIt\w*):[^\n]*\n(.*?)\n\.Lfunc_end", out.read_text(), re.S | re.M)
    return _instructions(m.group(2))


def test_accumulators_are_private(bf16_kernel):
    """The sums and the queries of the many-rows form lie in a0 .. a191, named by inline assembly: the compiler's own code
    never touches those."""
    own = {f"a{i}" for i in range(OWN_AGPRS)}
    for x in bf16_kernel:
        assert x.asm or not own & (x.dst | x.src), x.text
    used = set().union(*(x.dst | x.src for x in bf16_kernel if x.asm))
    assert own <= used


def test_products_wait_for_their_operands(bf16_kernel):
    """Products in inline assembly are not covered by the compiler's own waits: an operand that a vector instruction
    writes needs 2 states before the product reads it."""
    code, products = bf16_kernel, [x for x in bf16_kernel if x.asm and x.mfma]
    assert len(products) >= 90
    wanted = set().union(*(_registers(x.args[1]) | _registers(x.args[2]) for x in products))
    for i, w in enumerate(code):
        if w.mfma or not w.op.startswith("v_") or not w.dst & wanted:
            continue

        def visit(x, t):
            if x.asm and x.mfma:
                assert not w.dst & (_registers(x.args[1]) | _registers(x.args[2])), f"{w.text} -> {x.text} after {t}"
            return False
        _follow(code, i, 3, visit)


def test_results_are_read_late_enough(bf16_kernel):
    """... and a product's result needs 12 states (8 passes, 3, and 1 on gfx950) before anything but the product that adds
    to it reads or overwrites it."""
    code = bf16_kernel
    for i, w in enumerate(code):
        if not (w.asm and w.mfma):
            continue

        def visit(x, t):
            if x.mfma:
                if x.asm and _registers(x.args[0]) == w.dst and _registers(x.args[3]) in (w.dst, set()):
                    return True                            # goes on adding, or begins anew: checked from there
                hit = w.dst & (_registers(x.args[1]) | _registers(x.args[2]))
            else:
                hit = w.dst & (x.src | x.dst)
            assert not hit, f"{w.text} -> {x.text} after {t}"
            return False
        _follow(code, i, 12, visit)
