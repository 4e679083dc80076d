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
    assert attn(L, None, batch(width=16), **kw) == code and L.varrate_last_error()    # 1024 keys: may be cut


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
    assert need(1, 1, 8) == 0 and need(1, 1, 4, dtype=0) == 0
    assert 0 < need(1, 1, 9) <= need(1, 1, 64) < need(4, 4, 64) <= need(4, 4, 1 << 20)
    assert need(1 << 20, 1, 1 << 20) == need(1 << 22, 1, 1 << 20) == 2 * 256 * 256 * 130 * 4 + 16 + 256 * 40


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

struct Tile { int s = -1, g = 0, tile = 0; int64_t start = 0, w = 0; };
struct Share { int64_t pos; Tile t; bool inside; };
struct Piece { int s, g, tile; int32_t lo, hi; bool cut; int place; };

struct Call {
    std::vector<SeqRange> r;
    int G, Hg, causal, window;
    Costs c;
    Split split;
    int64_t head = 0;
    Line line(int s) const { return seq_line(r[s], Hg, causal, window, c); }
    Tile tile_of(int64_t pos) const {
        Tile t;
        t.g = (int)(pos / head);
        int64_t x = pos % head, base = t.g * head;
        for (int s = 0; s < (int)r.size(); ++s) {
            const Line l = line(s);
            const int64_t all = line_before(l, l.tiles);
            if (x < all) {
                t.s = s;
                t.tile = line_tile(l, x);
                CHECK(t.tile >= 0 && t.tile < l.tiles && line_before(l, t.tile) <= x && x < line_before(l, t.tile + 1));
                t.start = base + line_before(l, t.tile);
                t.w = line_at(l, t.tile);
                CHECK(t.w > 0 && t.start + t.w == base + line_before(l, t.tile + 1));
                return t;
            }
            x -= all;
            base += all;
        }
        CHECK(!"found");
        return t;
    }
    int64_t share_at(int i, Tile& t) const {
        const int64_t total = head * G, pos = share_begin(total, i, split);
        CHECK(pos >= 0 && pos <= total);
        if (pos >= total) return total;
        t = tile_of(pos);
        return t.start + cut_at(pos - t.start, t.w, is_many(r[t.s], Hg), c);
    }
};

// every tile's keys are some share's exactly once, and the second launch finds the pieces of those that were cut
static void shares_of(Call k, Split split) {
    const int among = split.among;
    k.split = split;
    k.head = 0;
    for (int s = 0; s < (int)k.r.size(); ++s) k.head += line_before(k.line(s), k.line(s).tiles);
    std::vector<Share> shares(among);
    std::vector<Piece> all;
    for (int i = 0; split.same && i < among; ++i) {        // every tile in equal pieces
        int u = i / split.same, x = i % split.same, each = among / split.same / k.G, in = u % each;
        Tile t;
        t.g = u / each;
        for (t.s = 0; in >= seq_tiles(k.r[t.s], k.Hg); ++t.s) in -= seq_tiles(k.r[t.s], k.Hg);
        const SeqRange r = k.r[t.s];
        t.tile = seq_tiles(r, k.Hg) - 1 - in;
        t.start = (int64_t)u * split.same;
        const int bm = tile_rows(r, k.Hg);
        const int32_t row0 = t.tile * bm, rows = (int32_t)std::min<int64_t>(bm, seq_rows(r, k.Hg) - row0);
        int32_t lo, hi;
        tile_keys(r, row0, rows, k.Hg, k.causal, k.window, lo, hi);
        piece_keys(x, x + 1, split.same, lo, hi);
        shares[i] = Share{i, t, x != 0};
        all.push_back(Piece{t.s, t.g, t.tile, lo, hi, true, 2 * i});
    }
    auto order = [](const Piece& a, const Piece& b) {
        return a.g != b.g ? a.g < b.g : a.s != b.s ? a.s < b.s : a.tile < b.tile;
    };
    std::stable_sort(all.begin(), all.end(), order);
    for (int i = 0; !split.same && i < among; ++i) {
        Tile t, last;
        const int64_t end = k.share_at(i + 1, last);
        int64_t pos = k.share_at(i, t);
        CHECK(i == 0 ? pos == 0 : pos <= end);
        shares[i] = Share{pos, t, pos > t.start && pos < t.start + t.w};
        for (int place = 2 * i; pos < end; place |= 1) {
            if (pos >= t.start + t.w) t = k.tile_of(pos);
            const int64_t x0 = pos - t.start, x1 = std::min(end - t.start, t.w);
            const SeqRange r = k.r[t.s];
            const int bm = tile_rows(r, k.Hg);
            const int32_t row0 = t.tile * bm, rows = (int32_t)std::min<int64_t>(bm, seq_rows(r, k.Hg) - row0);
            int32_t lo, hi;
            CHECK(rows > 0);
            tile_keys(r, row0, rows, k.Hg, k.causal, k.window, lo, hi);
            const bool cut = x1 - x0 != t.w;
            if (cut) piece_keys(x0, x1, t.w, lo, hi);
            CHECK(lo >= 0 && lo <= hi && hi <= (r.klen > lo ? r.klen : lo));
            all.push_back(Piece{t.s, t.g, t.tile, lo, hi, cut, place});
            pos = t.start + x1;
        }
    }
    // in the order of the shares a tile's pieces follow each other
    size_t at = 0, cuts = 0, joined = 0;
    for (int g = 0; g < k.G; ++g)
        for (int s = 0; s < (int)k.r.size(); ++s)
            for (int tile = 0; tile < seq_tiles(k.r[s], k.Hg); ++tile) {
                const SeqRange r = k.r[s];
                const int bm = tile_rows(r, k.Hg);
                const int32_t row0 = tile * bm, rows = (int32_t)std::min<int64_t>(bm, seq_rows(r, k.Hg) - row0);
                int32_t lo, hi, from = 0;
                tile_keys(r, row0, rows, k.Hg, k.causal, k.window, lo, hi);
                for (int i = 0; i < rows; i += rows > 40 ? 13 : 1) {       // no row sees keys outside
                    int32_t a, b;
                    row_keys(r, (row0 + i) / k.Hg, k.causal, k.window, a, b);
                    CHECK(b <= a || (a >= lo && b <= hi));
                }
                bool some = false;
                size_t n = 0;
                for (; at < all.size() && all[at].s == s && all[at].g == g && all[at].tile == tile; ++at, ++n) {
                    if (all[at].hi > all[at].lo) {
                        CHECK(all[at].lo == (some ? from : lo) && (!some || from % 64 == 0));
                        from = all[at].hi;
                        some = true;
                    }
                    CHECK(n == 0 || all[at].cut);
                }
                CHECK(n >= 1 && (hi <= lo || (some && from == hi)));
                CHECK((n > 1) == all[at - 1].cut);
                cuts += n > 1;
            }
    CHECK(at == all.size());
    for (int i = 1; i < among; ++i) {
        if (!shares[i].inside || (shares[i - 1].inside && shares[i - 1].t.start == shares[i].t.start)) continue;
        const Tile t = shares[i].t;
        int np = 2;
        while (i + np - 1 < among && shares[i + np - 1].inside && shares[i + np - 1].t.start == t.start) ++np;
        std::vector<int> places = {2 * (i - 1) + (shares[i - 1].pos == t.start ? 0 : 1)}, want;
        for (int p = 1; p < np; ++p) places.push_back(2 * (i + p - 1));
        for (const Piece& p : all)
            if (p.s == t.s && p.g == t.g && p.tile == t.tile) want.push_back(p.place);
        CHECK(places == want);
        ++joined;
    }
    CHECK(joined == cuts);
    std::vector<int> used;
    for (const Piece& p : all) if (p.cut) used.push_back(p.place);
    std::sort(used.begin(), used.end());
    CHECK(std::adjacent_find(used.begin(), used.end()) == used.end() && (used.empty() || used.back() < 2 * among));
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
        Call k{r, G, Hg, causal, window, c, Split{0, 0}, 0};
        const int n = max_groups(T, S, G, Hg, cap, c.lmin);
        const Split split = n ? split_of(s, n, c) : Split{0, 0};
        CHECK(n % 8 == 0 && n >= 0 && n <= SLOTS && split.among >= 0 && split.among <= n && split.among != 1);
        CHECK(split.same == 0 || (split.same > 1 && split.among == s.units * split.same));
        const int64_t records = max_records(T, S, G, Hg, cap, c.lmin);
        CHECK(records == 0 || (records == 2 * n * place_rows(T, Hg) && records <= 2 * SLOTS * ROWS_MANY));
        for (const SeqRange& x : r) CHECK(T * Hg > ROWS_FEW || seq_rows(x, Hg) <= ROWS_FEW || !rising);
        if (s.head > 0 && s.units < 20000) {
            if (split.among) shares_of(k, split);
            shares_of(k, Split{pick_of(2, 256), 0});
            shares_of(k, Split{2, 0});
            if (s.units <= 128) shares_of(k, Split{(int32_t)s.units * 2, 2});
            if (s.units <= 36) shares_of(k, Split{(int32_t)s.units * 7, 7});
        }
        if (rising) CHECK(s.units <= max_units(T, S, G, Hg));
    }
    // the longest: nothing overflows
    for (int bf = 0; bf < 2; ++bf) {
        const Costs c = costs_of(bf);
        const SeqRange r = seq_range(0, 1 << 20, 1 << 30, 1 << 20, 1 << 30);
        const Line l = seq_line(r, 1024, 1, 0, c);
        const int64_t all = line_before(l, l.tiles);
        CHECK(all > 0 && all < (int64_t)1 << 60 && line_tile(l, all - 1) == l.tiles - 1 && line_tile(l, 0) == 0);
        for (int i = 1; i < 1000; ++i) {
            const int64_t x = all / 1000 * i;
            const int32_t t = line_tile(l, x);
            CHECK(line_before(l, t) <= x && x < line_before(l, t + 1));
        }
        int32_t lo = 0, hi = 1 << 30;
        piece_keys(line_at(l, 5) / 3, line_at(l, 5), line_at(l, 5), lo, hi);
        CHECK(lo % 64 == 0 && lo > (1 << 30) / 4 && hi == 1 << 30);
        Sums s;
        for (int i = 0; i < 65536; ++i) sum_up(s, SeqRange{0, 1 << 20, 1 << 30}, 1, 1024, 1, 0, c);
        CHECK(split_of(s, 256, c).among == 0);                // starts that fall: sums that could overflow are not divided
    }
    for (int among : {2, 7, 8, 9, 100, 255, 256}) {
        std::vector<int> hit(among + 1, 0);
        for (uint32_t b = 0; b < 256; ++b) ++hit[share_of(b, among)];
        for (int i = 0; i < among; ++i) CHECK(hit[i] == 1);
    }
    // every whole tile of a call is one workgroup's, forwards and backwards
    for (uint32_t n : {8u, 16u, 248u, 256u})
        for (int rounds : {1, 2, 5}) {
            std::vector<int> hit(n * rounds, 0);
            for (uint32_t b = 0; b < n; ++b)
                for (int k = 0; k < rounds; ++k) {
                    const int64_t i = tile_number(b, n, b & 8 ? rounds - 1 - k : k);
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
