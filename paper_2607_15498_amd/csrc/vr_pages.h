// Index arithmetic of the paged cache, shared by the kernels and by a host build of it (the tests
// walk it on the CPU).  Everything that a kernel follows out of device memory (starts, lengths,
// page numbers) goes through here and is brought into range first: a bad entry costs its own
// tokens, never an access outside the buffers.
#pragma once
#include <math.h>
#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define VR_HD __host__ __device__ __forceinline__
#else
#define VR_HD static inline
#endif

namespace vr {

constexpr int PAGE_MIN = 16, PAGE_MAX = 256;   // powers of two

// The rows [q0, q0 + qlen) of the packed new tokens and the cached length of one sequence.
struct SeqRange { int32_t q0, qlen, klen; };

VR_HD int32_t clamp_i32(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// T packed rows; cap = table width x page size, the longest sequence that the table can hold
VR_HD SeqRange seq_range(int32_t start, int32_t end, int32_t len, int32_t T, int32_t cap) {
    SeqRange r;
    r.q0 = clamp_i32(start, 0, T);
    r.qlen = clamp_i32(end, r.q0, T) - r.q0;
    r.klen = clamp_i32(len, 0, cap);
    return r;
}

// The sequence of packed row i: the last s with q_start[s] <= i, -1 when i lies before the first
// or behind the last sequence (empty sequences have no rows and are passed over).
VR_HD int find_seq(const int32_t* q_start, int S, int32_t i) {
    if (i < q_start[0] || i >= q_start[S]) return -1;
    int lo = 0, hi = S;                        // q_start[lo] <= i < q_start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (q_start[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A page number of the table, or -1 when it names no page of the pool.
VR_HD int32_t good_page(int32_t page, int32_t n_pages) { return page >= 0 && page < n_pages ? page : -1; }

// ---- how the attention is cut ----------------------------------------------------------------
// The rows of one (sequence, KV head) are its qlen x Hg (new token, query head) pairs, token-major.
// Up to ROWS_FEW of them make one tile, whose keys a workgroup's waves divide among themselves; more
// are cut into tiles of ROWS_MANY rows, which the waves divide.  A call is shared out in one of three ways:
// whole tiles, one of each round of workgroups to each; every tile in the same number of pieces, one a workgroup; or all
// work laid end to end (head after head, its sequences, their tiles, a tile's keys) and divided evenly, so that a
// workgroup has the end of one tile, whole tiles and the beginning of another.  The second launch joins the tiles
// that were cut.
constexpr int ROWS_FEW = 32, ROWS_MANY = 256;
constexpr int SLOTS = 256;                     // workgroups that the card holds at once (one per CU)

VR_HD int64_t seq_rows(SeqRange r, int Hg) { return (int64_t)r.qlen * Hg; }
VR_HD int tile_rows(SeqRange r, int Hg) { return seq_rows(r, Hg) <= ROWS_FEW ? ROWS_FEW : ROWS_MANY; }
VR_HD int32_t seq_tiles(SeqRange r, int Hg) {
    const int bm = tile_rows(r, Hg);
    return (int32_t)((seq_rows(r, Hg) + bm - 1) / bm);
}
// the most keys that one of the sequence's tiles sees, counted from a multiple of 64
VR_HD int32_t seq_span(SeqRange r, int Hg, int window) {
    if (!window) return r.klen;
    const int64_t n = window + 63 + (tile_rows(r, Hg) + Hg - 2) / Hg;     // the tile's last token is that far from its first
    return n < r.klen ? (int32_t)n : r.klen;
}
// Costs, in units of 8 cycles of a workgroup, as measured: per key of a tile of few rows while all
// workgroups read (the memory's share) and of one of many rows (the matrix cores'); of a piece's start
// and end, of few rows and of many; and of joining tiles in the second launch (what it takes beyond being there),
// which besides reads what the first has written: JOIN_UNIT partial rows (1040 bytes each, both ways) cost 1.
constexpr int JOIN_UNIT = 16;
struct Costs { int32_t few, many, piece_few, piece_many, join, lmin; };      // lmin: shortest piece, keys
VR_HD Costs costs_of(bool bf16) {
    return bf16 ? Costs{5, 8, 600, 4400, 400, 256} : Costs{12, 72, 600, 1800, 400, 128};
}
VR_HD bool is_many(SeqRange r, int Hg) { return seq_rows(r, Hg) > ROWS_FEW; }

// The cost of a sequence's tiles for one head: a + b (t + 1) for tile t.  (Tiles of causal chunks see 256 / Hg keys more
// one after another; what is rounded in b shifts a little work, and nothing else hangs on it.)
struct Line { int64_t a, b; int32_t tiles; };
VR_HD Line seq_line(SeqRange r, int Hg, int causal, int window, Costs c) {
    const int32_t tiles = seq_tiles(r, Hg), first = r.klen - r.qlen;       // keys before the new tokens
    const bool many = is_many(r, Hg);
    const int64_t piece = many ? c.piece_many : c.piece_few, cost = many ? c.many : c.few;
    if (many && causal && !window && first >= 0) return Line{piece + cost * first, ROWS_MANY * cost / Hg, tiles};
    return Line{piece + cost * seq_span(r, Hg, window), 0, tiles};
}
// cost of the tiles before tile t
VR_HD int64_t line_before(const Line& l, int64_t t) { return t * l.a + l.b * (t * (t + 1) / 2); }
VR_HD int64_t line_at(const Line& l, int64_t t) { return l.a + l.b * (t + 1); }
// the tile that `x` (of all tiles' cost) falls into: about, then exactly
VR_HD int32_t line_tile(const Line& l, int64_t x) {
    if (l.tiles <= 1) return 0;
    float t;
    if (l.b == 0) t = (float)x / (float)l.a;
    else {
        const float m = (float)l.a + 0.5f * (float)l.b;
        t = (sqrtf(m * m + 2.f * (float)l.b * (float)x) - m) / (float)l.b;
    }
    int64_t i = t < (float)l.tiles ? (int64_t)t : l.tiles;
    if (i > l.tiles - 1) i = l.tiles - 1;
    while (i > 0 && line_before(l, i) > x) --i;
    while (i < l.tiles - 1 && line_before(l, i + 1) <= x) ++i;
    return (int32_t)i;
}
// A cut at x of a tile of cost w: where it leaves too little on either side (few rows: the shortest piece; many: 64 keys, and
// what a piece's start and end cost), at the nearer end instead.
VR_HD int64_t cut_at(int64_t x, int64_t w, bool many, Costs c) {
    const int64_t keys = many ? 64 * (int64_t)c.many : (int64_t)c.lmin * c.few;
    const int64_t least = many && keys < c.piece_many ? c.piece_many : keys;
    return x >= least && w - x >= least ? x : 2 * x < w ? 0 : w;
}
// ... and how many of the tile's `all` keys lie before it
VR_HD int32_t cut_key(int64_t x, int64_t w, int32_t all) {
    if (x >= w) return all;
    const float k = (float)all * ((float)x / (float)w) + 32.f;
    return k < (float)all ? (int32_t)k & ~63 : all & ~63;
}

// What the choice needs of the sequences.  The floats bound sums that could overflow (of starts that fall).
struct Sums {
    uint64_t head = 0;                         // cost of one head's work
    int64_t units = 0;                         // tiles x heads
    float total = 0.f, many = 0.f, units_many = 0.f, longest = 0.f;
};
VR_HD void sum_up(Sums& t, SeqRange r, int G, int Hg, int causal, int window, Costs c) {
    const Line l = seq_line(r, Hg, causal, window, c);
    const int64_t all = line_before(l, l.tiles);
    t.head += (uint64_t)all;
    t.units += (int64_t)l.tiles * G;
    t.total += (float)all * (float)G;
    if (is_many(r, Hg)) {
        t.many += (float)all * (float)G;
        t.units_many += (float)l.tiles * (float)G;
    }
    const float last = l.tiles ? (float)line_at(l, l.tiles - 1) : 0.f;
    if (last > t.longest) t.longest = last;
}
// How n workgroups share the work out: into `among` shares (0: whole tiles), `same` to every tile (0: even ones).
// What is estimated to take the shortest.  Each forced, us (bf16, 8 KV heads of 4, unless said otherwise):
//                                                  whole    equal    even
//   2048 tokens over 32768 (256 tiles, alike)        966              1010
//   8192 tokens from the first (1024 tiles)          547               635
//   1003 over 5003 (128 tiles, alike)                158      109      124
//   1 over 32768 (8 tiles)                           439       35       36
//   16 of 1 over 301 .. 8146                         144       85       77
//   32 of 1 over 100 .. 21800                        402      349      287
//   fp32 prompts of 1531 and 777 (296 tiles)         406      409      257
struct Split { int32_t among, same; };
VR_HD Split split_of(const Sums& s, int n, Costs c) {
    const Split tiles = {0, 0};
    if (!(s.total > 0.f && s.total < 1e18f)) return tiles;
    const float units = (float)s.units, all = (float)n, turns = units / all, mean = s.total / units;
    const float piece = (float)(s.many > 0.f ? c.piece_many : c.piece_few), tile = (float)(ROWS_MANY / JOIN_UNIT);
    // one round of `pieces` whose longest is `x`: few rows share the memory, down to about half of the cost for a lone one
    // (1024 instead of 256 keys: 12.5 ns a key)
    auto round_of = [&](float pieces, float x) {
        const float load = s.many > 0.f ? 1.f : pieces < 0.55f * all ? 0.55f : pieces / all;
        return (x - piece) * load + piece;
    };
    const float rounds = (float)((s.units + n - 1) / n);
    float least_time = round_of(units, s.longest);
    if (rounds > 1.f) {                        // tiles one to each, in turned order: what the last round lacks
        least_time = s.total / all + (rounds - turns) * mean;
        const float odd = s.total / all + 0.5f * (s.longest - mean);
        if (((int64_t)rounds & 1) && least_time < odd) least_time = odd;
    }
    Split best = tiles;
    // shares no shorter than a shortest piece on average
    const float shortest = (float)((s.many > 0.f ? c.many : c.few) * c.lmin);
    const float among = s.total < (shortest + piece) * all ? (float)(int32_t)(s.total / (shortest + piece)) : all;
    if (among >= 2.f) {
        const float cuts = among * (s.many / s.total);
        const float x = round_of(among, s.total / among) + piece + (float)c.join +
                        tile * (cuts + (s.units_many < cuts ? s.units_many : cuts));
        if (x < least_time) {
            least_time = x;
            best.among = (int32_t)among;
        }
    }
    // every tile in the same number of pieces
    const float fit = (s.longest - piece) / shortest;
    int32_t same = s.units < n ? n / (int32_t)s.units : 0;
    if (fit < (float)same) same = (int32_t)fit;
    if (same > 1) {
        const float x = round_of(units * (float)same, (s.longest - piece) / (float)same + piece) + (float)c.join +
                        tile * s.units_many * (float)same;
        if (x < least_time) best = Split{(int32_t)s.units * same, same};
    }
    return best;
}
// where share i begins (that all workgroups get the same number is what counts)
VR_HD int64_t share_begin(int64_t total, int32_t i, Split p) {
    return i >= p.among ? total : (int64_t)((float)total * ((float)i / (float)p.among));
}
// Workgroup b's share (`among`: none).  Workgroups b, b + 8, .. run on one die, whose L2 they share, and get shares side
// by side, so that a head's keys are read into few dies' caches.
VR_HD int32_t share_of(uint32_t b, int32_t among) {
    const int32_t each = (among + 7) >> 3, i = (int32_t)(b >> 3);
    const int32_t share = (int32_t)(b & 7u) * each + i;
    return i < each && share < among ? share : among;
}

// most (tile, head) pairs of any call with T rows and S sequences; workgroups that a call whose tables hold `cap` tokens can use
VR_HD int64_t max_units(int64_t T, int S, int G, int Hg) { return G * (T * Hg / ROWS_MANY + (S < T ? S : T)); }
// Those of a call, none where they are more: then starts fall (rows belong to several sequences, up to S / 2 times as much
// work as any call has), and nothing is computed.
VR_HD int64_t units_of(int64_t units, int64_t most) { return units <= most ? units : 0; }
VR_HD int max_groups(int64_t T, int S, int G, int Hg, int64_t cap, int lmin) {
    const int64_t n = max_units(T, S, G, Hg) * ((cap + lmin - 1) / lmin);
    return n < SLOTS ? (int)((n + 7) & ~(int64_t)7) : SLOTS;
}
// Partial results: a workgroup has two places, for a tile that it begins with and for one that it ends with.
VR_HD int place_rows(int64_t T, int Hg) { return T * Hg <= ROWS_FEW ? ROWS_FEW : ROWS_MANY; }
VR_HD int64_t max_records(int64_t T, int S, int G, int Hg, int64_t cap, int lmin) {
    return cap <= 2 * lmin ? 0 : (int64_t)2 * max_groups(T, S, G, Hg, cap, lmin) * place_rows(T, Hg);
}

// Keys [lo, hi) that the sequence's new token i sees (none when hi <= lo).
VR_HD void row_keys(SeqRange r, int32_t i, int causal, int window, int32_t& lo, int32_t& hi) {
    const int32_t pos = r.klen - r.qlen + i;
    hi = causal ? (pos + 1 < r.klen ? pos + 1 : r.klen) : r.klen;
    if (hi < 0) hi = 0;
    lo = window && pos - window + 1 > 0 ? pos - window + 1 : 0;
}
// Keys [lo, hi) of a tile's rows row0 .. row0 + rows - 1 ...
VR_HD void tile_keys(SeqRange r, int32_t row0, int32_t rows, int Hg, int causal, int window, int32_t& lo, int32_t& hi) {
    int32_t x;
    row_keys(r, row0 / Hg, causal, window, lo, x);
    row_keys(r, (row0 + rows - 1) / Hg, causal, window, x, hi);
    if (hi < lo) hi = lo;
}
// ... and of them those of the piece [x0, x1) of its cost w: cuts lie at multiples of 64 keys
VR_HD void piece_keys(int64_t x0, int64_t x1, int64_t w, int32_t& lo, int32_t& hi) {
    const int32_t from = lo & ~63, all = hi - from;
    const int32_t k0 = from + cut_key(x0, w, all), k1 = from + cut_key(x1, w, all);
    if (k0 > lo) lo = k0;
    if (k1 < hi) hi = k1;
    if (hi < lo) hi = lo;
}
// Whole tiles: the number of the (tile, head) pair that workgroup b of n (a multiple of 8) takes in a round: b, then in
// turned order (a sequence's tiles shrink along its numbers; turning gives every workgroup long and short
// ones), b % 8 kept: heads stay on their die's L2.
VR_HD int64_t tile_number(uint32_t b, uint32_t n, int round) {
    return (int64_t)round * n + (round & 1 ? ((n - 1 - b) & ~7u) | (b & 7u) : b);
}

}  // namespace vr
