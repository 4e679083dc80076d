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
// The rows of one (sequence, KV head) are its qlen x Hg (new token, query head) pairs, token-major,
// in tiles of BM rows; the keys that any of the sequence's rows sees, [first, klen), are cut into
// pieces of L tokens.  L is one number for the whole call, so that long sequences get more pieces.
struct Cut { int64_t units; int64_t L; };      // units: (sequence, tile) pairs; L: tokens per piece

VR_HD int32_t seq_tiles(SeqRange r, int Hg, int BM) { return (int32_t)(((int64_t)r.qlen * Hg + BM - 1) / BM); }
// first key that the sequence's first row sees, at a multiple of 64
VR_HD int32_t seq_first(SeqRange r, int window) {
    if (!window) return 0;
    const int64_t f = (int64_t)r.klen - r.qlen - window + 1;
    return f > 0 ? (int32_t)(f < r.klen ? f : r.klen) & ~63 : 0;
}
VR_HD int32_t seq_span(SeqRange r, int window) { return r.klen - seq_first(r, window); }
// piece length from the sums over the sequences of tiles and tiles x span: about `target` pieces
// over all G heads, none shorter than lmin; without splitting when there are units enough
VR_HD int64_t cut_len(int64_t units, int64_t work, int G, int target, int lmin) {
    if (units * G >= target) return INT64_MAX / 2;
    const int64_t per = (work * G + target - 1) / target;
    const int64_t L = (per + 127) / 128 * 128;
    return L < lmin ? lmin : L;
}
VR_HD int32_t seq_pieces(int32_t span, int64_t L) {
    return span <= L ? 1 : (int32_t)((span + L - 1) / L);
}
// most (unit, head, piece) triples of any call with T rows and S sequences
VR_HD int64_t max_pieces(int64_t T, int S, int G, int Hg, int BM, int target, int64_t cap, int lmin) {
    const int64_t units = G * (T * Hg / BM + (S < T ? S : T));
    const int64_t most = units * ((cap + lmin - 1) / lmin);   // no piece is shorter than lmin
    return units + target < most ? units + target : most;
}

// Keys [lo, hi) that row `row` of the sequence sees (none when hi <= lo).
VR_HD void row_keys(SeqRange r, int32_t i, int causal, int window, int32_t& lo, int32_t& hi) {
    const int32_t pos = r.klen - r.qlen + i;
    hi = causal ? (pos + 1 < r.klen ? pos + 1 : r.klen) : r.klen;
    if (hi < 0) hi = 0;
    lo = window && pos - window + 1 > 0 ? pos - window + 1 : 0;
}

}  // namespace vr
