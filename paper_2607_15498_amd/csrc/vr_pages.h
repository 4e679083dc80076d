// Index arithmetic of the paged cache, shared by the kernels and by a host build of it (the tests
// walk it on the CPU).  Everything that a kernel follows out of device memory (starts, lengths,
// page numbers) goes through here and is brought into range first: a bad entry costs its own
// tokens, never an access outside the buffers.
#pragma once
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
// are cut into tiles of ROWS_MANY rows, which the waves divide.  The keys that a
// tile sees are cut into pieces, the same number and length for all tiles of a sequence, of a cost of
// about L at most: one number for the whole call, so that long sequences get more pieces.  (Tiles that
// see fewer keys have empty pieces at the end.)
constexpr int ROWS_FEW = 32, ROWS_MANY = 256;
constexpr int SLOTS = 256;                     // workgroups that the card holds at once (one per CU)
constexpr int32_t WHOLE = INT32_MAX;           // L of a call that is not cut

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
// the keys that its tiles see on average
VR_HD int32_t seq_mean(SeqRange r, int32_t span, int causal) {
    const int32_t first = r.klen - r.qlen > 0 ? r.klen - r.qlen : 0;       // keys before the new tokens
    return causal && span == r.klen ? first + (r.klen - first) / 2 + 1 : span;
}

// Costs, in units of 16 cycles of a workgroup, as measured: per key of a tile of few rows while all
// workgroups read (the memory's share) and of one of many rows (the matrix cores'); of a piece's start
// and end, and of the second launch, which besides reads what the first has written: JOIN_UNIT partial rows
// (1040 bytes each, both ways) cost 1.  A lone workgroup's few rows cost a quarter.
constexpr int JOIN_UNIT = 32;
struct Costs { int32_t few, many, piece, join, lmin; };      // lmin: shortest piece, keys (a power of two)
VR_HD Costs costs_of(bool bf16) {
    return bf16 ? Costs{4, 4, 400, 600, 256} : Costs{7, 36, 400, 600, 128};
}
VR_HD int32_t key_cost(SeqRange r, int Hg, Costs c) { return tile_rows(r, Hg) == ROWS_FEW ? c.few : c.many; }
// pieces of a span of keys at `cost` each (32-bit divisions: the plan's code is run once, and what it costs is
// fetching it)
VR_HD int32_t seq_pieces(int32_t span, int32_t cost, int32_t L, int32_t lmin) {
    if (L == WHOLE || span <= lmin) return 1;
    const uint64_t all = (uint64_t)(uint32_t)span * (uint32_t)cost;
    const uint32_t n = ((uint32_t)(all < (1u << 30) ? all : 1u << 30) + (uint32_t)L - 1) / (uint32_t)L;
    const uint32_t most = ((uint32_t)span + (uint32_t)lmin - 1) >> __builtin_ctz((uint32_t)lmin);
    return (int32_t)(n < most ? n : most);
}
// keys of each of a span's np pieces
VR_HD int32_t piece_len(int32_t span, int np) {
    return np == 1 ? span : (int32_t)((((uint32_t)span + (uint32_t)np - 1) / (uint32_t)np + 63) & ~63u);
}

// How many pieces: the cut with the shortest estimated time.  Candidate 0 is uncut; the others aim at 3/4
// of a piece for every slot (room for what rounding up adds), at 1, 2, 3 and 4.
constexpr int CUTS = 6;
constexpr int PIECES_MAX = 4 * SLOTS;          // of a cut call (an uncut one may have any number)
// spans: sum of tiles x span x cost over sequences and heads
VR_HD int32_t cut_try(int i, float spans) {
    if (i == 0) return WHOLE;
    const float slot = spans * (1.f / SLOTS);
    const float x = i == 1 ? slot * 4.f / 3.f : slot / (float)(i - 1);
    return x < 1e9f ? (int32_t)x + 1 : 1000000000;
}
// What the estimate needs of the sequences: first these sums (in floats: one instruction each, and only the
// choice hangs on them) ...
struct Sums { int64_t units = 0; float work = 0.f, spans = 0.f; int32_t longest = 0; bool many = false; };
VR_HD void sum_up(Sums& t, SeqRange r, int G, int Hg, int causal, int window, Costs c) {
    const int64_t n = (int64_t)seq_tiles(r, Hg) * G;
    const int32_t span = seq_span(r, Hg, window);
    const float cost = (float)n * (float)key_cost(r, Hg, c);
    t.units += n;
    t.work += cost * (float)seq_mean(r, span, causal);
    t.spans += cost * (float)span;
    if (n && span > t.longest) t.longest = span;
    t.many = t.many || tile_rows(r, Hg) != ROWS_FEW;
}
// ... then for every candidate these (counts up to 2^24 are exact, and PIECES_MAX is the most that is taken).
struct Cut { int32_t L; float pieces, partial, most; };   // partial: partial rows / JOIN_UNIT; most: cost of the longest piece
VR_HD Cut cut_begin(int i, float spans) { return Cut{cut_try(i, spans), 0.f, 0.f, 0.f}; }
VR_HD void cut_up(Cut& t, SeqRange r, int G, int Hg, int window, Costs c) {
    const int32_t tiles = seq_tiles(r, Hg), span = seq_span(r, Hg, window), cost = key_cost(r, Hg, c);
    const int32_t np = seq_pieces(span, cost, t.L, c.lmin);
    const float all = (float)G * (float)np, len = tiles ? (float)piece_len(span, np) * (float)cost : 0.f;
    t.pieces += all * (float)tiles;
    if (np > 1) t.partial += all * (float)seq_rows(r, Hg) * (1.f / JOIN_UNIT);
    if (len > t.most) t.most = len;
}
VR_HD float cut_cost(const Cut& t, const Sums& s, Costs c) {
    const float units = (float)s.units;
    if (t.pieces > units && t.pieces > (float)PIECES_MAX) return 1e30f;
    const float rounds = (float)(((int32_t)t.pieces + SLOTS - 1) / SLOTS);
    float cost = rounds * t.most;
    if (!s.many && t.pieces < (float)SLOTS) cost = t.most * (t.pieces < SLOTS / 4 ? SLOTS / 4 : t.pieces) * (1.f / SLOTS);
    // unlike pieces even out over several rounds (a sequence's longest come first)
    const float even = s.work * (1.f / SLOTS) + t.most;
    if (rounds > 1.f && cost > even) cost = even;
    return cost + rounds * (float)c.piece + (t.pieces > units ? (float)c.join + t.partial : 0.f);
}
struct Plan { int32_t L, pieces; };
VR_HD Plan uncut(const Sums& s) { return Plan{WHOLE, s.units < INT32_MAX ? (int32_t)s.units : INT32_MAX}; }
VR_HD bool may_cut(const Sums& s, Costs c) { return s.longest > c.lmin && s.units < PIECES_MAX; }

// Rows of many that a workgroup of the second launch joins: a half wave has 8 loads under way, of 4 rows' pieces or of 8
// pieces' rows.
VR_HD int join_rows(int np) { return np <= 4 ? 16 : 8; }

// most (tile, head) pairs and pieces of any call with T rows and S sequences whose tables hold `cap` tokens
VR_HD int64_t max_units(int64_t T, int S, int G, int Hg) { return G * (T * Hg / ROWS_MANY + (S < T ? S : T)); }
VR_HD int64_t max_pieces(int64_t T, int S, int G, int Hg, int64_t cap, int lmin) {
    const int64_t units = max_units(T, S, G, Hg);
    const int64_t most = units * ((cap + lmin - 1) / lmin);
    const int64_t cut = most < PIECES_MAX ? most : PIECES_MAX;
    return units > cut ? units : cut;
}
// most rows of partial results
VR_HD int64_t max_records(int64_t T, int S, int G, int Hg, int64_t cap, int lmin) {
    if (cap <= lmin) return 0;
    const int64_t p = max_pieces(T, S, G, Hg, cap, lmin);
    return (p < PIECES_MAX ? p : PIECES_MAX) * (T * Hg <= ROWS_FEW ? ROWS_FEW : ROWS_MANY);
}

// Keys [lo, hi) that the sequence's new token i sees (none when hi <= lo).
VR_HD void row_keys(SeqRange r, int32_t i, int causal, int window, int32_t& lo, int32_t& hi) {
    const int32_t pos = r.klen - r.qlen + i;
    hi = causal ? (pos + 1 < r.klen ? pos + 1 : r.klen) : r.klen;
    if (hi < 0) hi = 0;
    lo = window && pos - window + 1 > 0 ? pos - window + 1 : 0;
}
// Keys [lo, hi) of piece number `piece` of the np of the tile of rows row0 .. row0 + rows - 1 (none when hi <= lo): pieces start
// at multiples of 64, the first at the one before the tile's first key.
VR_HD void piece_keys(SeqRange r, int32_t row0, int32_t rows, int32_t piece, int32_t np, int Hg, int causal, int window,
                      int32_t& lo, int32_t& hi) {
    int32_t x;
    row_keys(r, row0 / Hg, causal, window, lo, x);
    row_keys(r, (row0 + rows - 1) / Hg, causal, window, x, hi);
    if (np == 1) return;
    const int32_t len = piece_len(seq_span(r, Hg, window), np);
    const int64_t p0 = (lo & ~63) + (int64_t)piece * len;
    if (lo < p0) lo = (int32_t)(p0 < r.klen ? p0 : r.klen);
    if (hi > p0 + len) hi = (int32_t)(p0 + len);
}
// The piece that workgroup b of n (a multiple of 8) takes in a round: b, then in turned order (the pieces of a sequence
// shrink along its numbers; turning gives every workgroup long and short ones), b % 8 kept: heads stay on their XCD's L2.
VR_HD int64_t piece_number(uint32_t b, uint32_t n, int round) {
    return (int64_t)round * n + (round & 1 ? ((n - 1 - b) & ~7u) | (b & 7u) : b);
}

}  // namespace vr
