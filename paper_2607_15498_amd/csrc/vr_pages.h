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
// and end, and of the second launch.  A lone workgroup's few rows cost a quarter.
struct Costs { int32_t few, many, piece, join, lmin; };      // lmin: shortest piece, keys
VR_HD Costs costs_of(bool bf16) {
    return bf16 ? Costs{4, 3, 400, 600, 256} : Costs{8, 40, 400, 600, 128};
}
VR_HD int32_t key_cost(SeqRange r, int Hg, Costs c) { return tile_rows(r, Hg) == ROWS_FEW ? c.few : c.many; }
// pieces of a span of keys at `cost` each
VR_HD int32_t seq_pieces(int32_t span, int32_t cost, int32_t L, int32_t lmin) {
    if (L == WHOLE || span <= lmin) return 1;
    const int64_t n = ((int64_t)span * cost + L - 1) / L, most = (span + lmin - 1) / lmin;
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
VR_HD int32_t cut_try(int i, int64_t spans) {
    if (i == 0) return WHOLE;
    const int64_t n = (int64_t)(i == 1 ? 3 : 4 * (i - 1)) * (SLOTS / 4), L = (spans + n - 1) / n;
    return L < 1 ? 1 : L < (1 << 30) ? (int32_t)L : 1 << 30;
}
// pieces: all of them; longest: the cost of the longest; work: of all; units: pieces of the uncut call; few: no
// sequence has many rows
VR_HD int64_t cut_cost(int64_t pieces, int64_t longest, int64_t work, int64_t units, bool few, Costs c) {
    if (pieces > units && pieces > PIECES_MAX) return INT64_MAX;
    const int64_t rounds = (pieces + SLOTS - 1) / SLOTS;
    int64_t t = rounds * longest;
    if (few && pieces < SLOTS) t = longest * (pieces < SLOTS / 4 ? SLOTS / 4 : pieces) / SLOTS;
    // unlike pieces even out over several rounds (a sequence's longest come first)
    if (rounds > 1 && t > work / SLOTS + longest) t = work / SLOTS + longest;
    return t + rounds * c.piece + (pieces > units ? c.join : 0);
}

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

// Keys [lo, hi) that row `row` of the sequence sees (none when hi <= lo).
VR_HD void row_keys(SeqRange r, int32_t i, int causal, int window, int32_t& lo, int32_t& hi) {
    const int32_t pos = r.klen - r.qlen + i;
    hi = causal ? (pos + 1 < r.klen ? pos + 1 : r.klen) : r.klen;
    if (hi < 0) hi = 0;
    lo = window && pos - window + 1 > 0 ? pos - window + 1 : 0;
}

}  // namespace vr
