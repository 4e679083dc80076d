// Attention of new tokens over a paged cache, gfx950.
//
// o_r = sum_t p_rt v_t / sum_t p_rt,  p_rt = exp(c (x_rt - max_t x_rt)),  x_rt = <q_r, k_t>, over the
// keys t that row r sees, in one pass with a running maximum and sum.  The rows of one KV head are the
// (new token, query head) pairs that read it.  Everything is computed transposed: S^T = K Q^T leaves
// a lane one row (query) and 16 keys of every 32, so maximum and sum are almost wholly within the
// lane, and S^T is already the B operand of O^T = V^T P^T (the keys' order in a product is free, and
// V^T's fragments are read in the order in which S^T holds them).
//
// Two forms.  Rows: a workgroup's 4 waves hold 32 rows each and share the key tiles (prompts and
// chunks; bound by the matrix cores).  Keys: the 4 waves share 32 rows and take every fourth key
// tile each, with rings of their own and no barrier, joined at the end (single tokens; bound by the
// reads of K and V).  When there are too few (sequence, head, row tile) units for the card, the keys
// are cut into pieces (vr_pages.h) and a second launch joins the pieces' partial rows.
//
// Keys and values come by direct-to-LDS loads of 1 KB (whole rows).  Row r's 16-byte piece c lies at
// place c ^ f(r), f(r) = 4 (r % 4) + (r / 4) % 4, which spreads the K fragment reads (32 rows, one
// piece) and the transposing V reads (8 rows, 4 pieces) over all banks.
#include "vr_internal.h"
#include "vr_pages.h"

namespace vr {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short pa_s16x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const void* q;
    void* out;
    const void* k;
    const void* v;
    const int32_t* table;
    const int32_t* kv_len;
    const int32_t* q_start;
    float* rec;                     // split calls: per piece [BM][128] sums, then all pieces' [BM][2] (max, sum)
    int64_t q_stride, out_stride;   // elements between tokens
    int64_t table_stride;
    int64_t rec_pieces;             // pieces that rec holds
    int32_t T, S, cap, n_pages, G, Hg, shift;
    int32_t causal, window, target, lmin;
    float c;                        // softmax scale x log2 e
};

// rows of a bad page: 1 KB of zeros
__device__ const uint4 pa_zeros[64] = {};

// wave-uniform 32-bit loads of the caller's tables through the scalar cache
typedef const __attribute__((address_space(4))) int32_t* const_i32;
__device__ __forceinline__ int32_t uload(const int32_t* p, int64_t i) {
    return ((const_i32)(uintptr_t)p)[i];
}

// One direct-to-LDS load: 16 bytes per lane from base + off to LDS byte address dst + 16 lane.
__device__ __forceinline__ void lds_load(const void* base, uint32_t off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(dst)
                 : "memory", "m0");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(float a, float b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// a value that all lanes hold, as a scalar
__device__ __forceinline__ int32_t first_lane(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t first_lane(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int32_t)(uint32_t)v);
    return (int64_t)((uint64_t)(uint32_t)first_lane((int32_t)(v >> 32)) << 32 | lo);
}

// ---- the call's cut, computed by every wave from the device lengths ----------------------------
__device__ __forceinline__ int64_t wave_sum(int64_t v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, WAVE);
    return v;
}
__device__ __forceinline__ SeqRange load_range(const AttnArgs& a, int s) {
    SeqRange r = {0, 0, 0};
    if (s < a.S) r = seq_range(a.q_start[s], a.q_start[s + 1], a.kv_len[s], a.T, a.cap);
    return r;
}
__device__ __forceinline__ Cut wave_cut(const AttnArgs& a, int BM) {
    const int lane = threadIdx.x & 63;
    int64_t units = 0, work = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const SeqRange r = load_range(a, s0 + lane);
        const int64_t t = seq_tiles(r, a.Hg, BM);
        units += t;
        work += t * seq_span(r, a.window);
    }
    Cut c;
    c.units = first_lane(wave_sum(units));
    c.L = cut_len(c.units, first_lane(wave_sum(work)), a.G, a.target, a.lmin);
    return c;
}
// The sequence of piece number idx: its pieces are (tile, piece, head) triples, heads innermost and the
// last tile first (with causal rows it sees the most keys).  base: the sequence's first number.
struct Unit { SeqRange r; int32_t s, np; int64_t base; };
template <typename F>
__device__ __forceinline__ bool scan_units(const AttnArgs& a, const Cut& cut, int BM, Unit& u, F&& pick) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const SeqRange r = load_range(a, s0 + lane);
        const int32_t np = seq_pieces(seq_span(r, a.window), cut.L);
        const int64_t n = (int64_t)seq_tiles(r, a.Hg, BM) * np * a.G;
        int64_t up = n;                        // inclusive scan over the lanes
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int64_t x = __shfl_up(up, m, WAVE);
            if (lane >= m) up += x;
        }
        const uint64_t hit = __ballot(pick(s0 + lane, before + up));
        if (hit) {
            const int l = __builtin_ctzll(hit);
            u.r.q0 = first_lane(__shfl(r.q0, l, WAVE));
            u.r.qlen = first_lane(__shfl(r.qlen, l, WAVE));
            u.r.klen = first_lane(__shfl(r.klen, l, WAVE));
            u.np = first_lane(__shfl(np, l, WAVE));
            u.base = first_lane(before + __shfl(up - n, l, WAVE));
            u.s = first_lane(s0 + l);
            return true;
        }
        before += first_lane(__shfl(up, 63, WAVE));
    }
    return false;
}

template <typename ET, bool KEYS>
struct Form {
    static constexpr bool BF = sizeof(ET) == 2;
    static constexpr int ROWB = D * (int)sizeof(ET);       // bytes of a row
    static constexpr int NK = !KEYS && BF ? 2 : 1;         // 32-key blocks per tile
    static constexpr int KT = 32 * NK;                     // keys per tile
    static constexpr int BM = KEYS ? 32 : 128;             // rows per workgroup
    static constexpr int KB = KT * ROWB;                   // bytes of a K (or V) tile
    static constexpr int NST = KEYS && !BF ? 1 : 2;        // tiles in a ring
    static constexpr int RING = NST * 2 * KB;              // [stage][K, V]
    static constexpr int JOIN = KEYS ? 4 * 32 * (132 + 2) * 4 : 0;
    static constexpr int RINGS = (KEYS ? 4 : 1) * RING;
    static constexpr size_t LDS = RINGS > JOIN ? RINGS : JOIN;
    static constexpr int CH = KEYS ? KB / 4096 : 1;        // 4 KB chunks that a wave brings of a K tile
    static constexpr int NU = BF ? 8 : 16;                 // 16-byte K fragments per lane and 32 keys
    static constexpr int QV = BF ? 8 : 16;
    static_assert(LDS <= 160 * 1024, "one workgroup fits a CU");
};

// 4 waves; see the head of the file.
template <typename ET, bool KEYS>
__global__ __launch_bounds__(256, KEYS ? 1 : 2) void paged_attn_kernel(AttnArgs a) {
    typedef Form<ET, KEYS> F;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int wave = first_lane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int l32 = lane & 31, h = lane >> 5;
    uint8_t* ring = smem + (KEYS ? wave * F::RING : 0);
    const uint32_t ring0 = first_lane((int)(uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)ring);
    const Cut cut = wave_cut(a, F::BM);
    const int G = a.G, Hg = a.Hg, shift = a.shift;
    const int64_t head_bytes = (int64_t)F::ROWB << shift;  // one head's rows of a page

    // load offsets: rows (lane / (ROWB / 16)) of a 1 KB piece, places permuted
    constexpr int PPR = F::ROWB / 16;
    const int lrow = lane / PPR;
    const uint32_t off0 = (uint32_t)(lrow * F::ROWB + ((lane % PPR) ^ ((lrow & 3) << 2)) * 16);
    // K fragment: row l32, piece 2 u + h
    const int kf = ((l32 & 3) << 2) | ((l32 >> 2) & 3);
    const uint32_t kaddr = (uint32_t)(l32 * F::ROWB + (h ^ kf) * 16);

    Unit u;
    int64_t end = -1;                                      // piece numbers below it are u's
    for (int64_t idx = blockIdx.x;; idx += gridDim.x) {
        if (idx >= end) {
            if (!scan_units(a, cut, F::BM, u, [&](int, int64_t upto) { return upto > idx; })) break;
            end = u.base + (int64_t)seq_tiles(u.r, Hg, F::BM) * u.np * G;
        }
        const SeqRange r = u.r;
        const int64_t in = idx - u.base;
        const int g = (int)(in % G);
        const int piece = (int)(in / G % u.np);
        const int tile = seq_tiles(r, Hg, F::BM) - 1 - (int)(in / G / u.np);
        const int32_t rows = (int32_t)((int64_t)r.qlen * Hg - (int64_t)tile * F::BM);   // rows from here on
        const int32_t row0 = tile * F::BM;
        const int32_t wrow0 = row0 + (KEYS ? 0 : 32 * wave);
        // keys that the workgroup's rows see, and of them this piece
        int32_t lo, hi, x;
        row_keys(r, row0 / Hg, a.causal, a.window, lo, x);
        row_keys(r, (row0 + (rows < F::BM ? rows : F::BM) - 1) / Hg, a.causal, a.window, x, hi);
        if (u.np > 1) {
            const int64_t p0 = seq_first(r, a.window) + piece * cut.L;
            if (lo < p0) lo = (int32_t)p0;
            if (hi > p0 + cut.L) hi = (int32_t)(p0 + cut.L);
        }
        lo = first_lane(lo);
        hi = first_lane(hi);
        // this lane's row, and the ranges of the wave's first and last row
        const int32_t nrow = rows - (wrow0 - row0);        // rows from the wave's first on
        const bool live = l32 < nrow;
        const int32_t myrow = wrow0 + (live ? l32 : 0);
        const int32_t tok = nrow > 0 ? myrow / Hg : 0;
        int32_t mylo, myhi, firsthi, lastlo, lasthi, firstlo;
        row_keys(r, tok, a.causal, a.window, mylo, myhi);
        row_keys(r, wrow0 / Hg, a.causal, a.window, firstlo, firsthi);
        row_keys(r, (wrow0 + (nrow < 32 ? nrow : 32) - 1) / Hg, a.causal, a.window, lastlo, lasthi);
        if (nrow <= 0) firstlo = lastlo = firsthi = lasthi = 0;
        // the row's query: B operand, 16-byte pieces 2 u + h
        u32x4 qf[F::QV];
        {
            const int64_t t = r.q0 + tok;
            const ET* src = (const ET*)a.q + t * a.q_stride + (int64_t)(g * Hg + (nrow > 0 ? myrow % Hg : 0)) * D;
#pragma unroll
            for (int k = 0; k < F::QV; ++k) qf[k] = load16((const uint8_t*)src + (2 * k + h) * 16);
        }
        float m = -INFINITY, l = 0.f;
        f32x16 acc[4];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

        const int32_t* trow = a.table + (int64_t)u.s * a.table_stride;
        const int32_t t_first = lo & ~(F::KT - 1);
        const int32_t step = KEYS ? 4 * F::KT : F::KT;
        const uint8_t* kbase = (const uint8_t*)a.k + (int64_t)g * head_bytes;
        const uint8_t* vbase = (const uint8_t*)a.v + (int64_t)g * head_bytes;
        constexpr int NG = F::KT / 16;
        // pages of the next tile to bring: of this wave's chunks, and which 16-key groups have one
        int32_t page[F::CH];
        uint32_t gm_next = 0;
        auto page_at = [&](int32_t t) {
            const int32_t p = uload(trow, (t < r.klen ? t : r.klen - 1) >> shift);
            return first_lane(t < r.klen ? good_page(p, a.n_pages) : -1);
        };
        auto fetch_pages = [&](int32_t t0) {
#pragma unroll
            for (int c = 0; c < F::CH; ++c) page[c] = page_at(t0 + (KEYS ? c : wave) * (4096 / F::ROWB) / 16 * 16);
            gm_next = 0;
#pragma unroll
            for (int j = 0; j < NG; ++j) gm_next |= (page_at(t0 + 16 * j) >= 0 ? 1u : 0u) << j;
        };
        // this wave's share of tile t0's keys (or values) into LDS at dst
        auto bring = [&](const uint8_t* pool, int32_t t0, uint32_t dst) {
#pragma unroll
            for (int c = 0; c < F::CH; ++c) {
                const int ch = KEYS ? c : wave;
                const int crow = ch * (4096 / F::ROWB);
                const int32_t p = page[c];
                const int32_t slot = (t0 + crow) & ((1 << shift) - 1);
                const uint8_t* src = (const uint8_t*)first_lane(
                    (int64_t)(p >= 0 ? pool + (int64_t)p * G * head_bytes + (int64_t)slot * F::ROWB : (const uint8_t*)pa_zeros));
                const int adv = p >= 0 ? 1024 : 0;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    // rows 4 v + .. (bf16) or 2 v + .. (fp32) of the chunk: the rest of f(row)
                    const uint32_t fx = F::BF ? (uint32_t)v & 3u : (uint32_t)(((v & 1) << 3) | (((v >> 1) + 2 * (ch & 1)) & 3));
                    lds_load(src + v * adv, off0 ^ (fx << 4), dst + ch * 4096 + v * 1024);
                }
            }
        };
        // rows of the last page behind the sequence's end: their values are not read as data
        auto clear_tail = [&](int32_t t0, uint8_t* vt) {
            const int32_t from = r.klen - t0;              // first such row of the tile
            if (from >= F::KT || (from & 15) == 0) return;
            const int32_t to = (from + 15) & ~15;
            for (int i = lane; i < (to - from) * PPR; i += 64) {
                const int row = from + i / PPR;
                if (KEYS || row / (4096 / F::ROWB) == wave)
                    *reinterpret_cast<uint4*>(vt + row * F::ROWB + (i % PPR) * 16) = uint4{0, 0, 0, 0};
            }
        };

        // one tile: scores, running maximum and sum, value products
        f32x16 sc[F::NK];
        auto scores = [&](const uint8_t* kt) {
#pragma unroll
            for (int n = 0; n < F::NK; ++n) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[n][i] = 0.f;
#pragma unroll
                for (int k = 0; k < F::NU; ++k) {
                    const u32x4 f = *reinterpret_cast<const u32x4*>(kt + 32 * n * F::ROWB + (kaddr ^ (32u * k)));
                    if constexpr (F::BF) sc[n] = mfma32(f, qf[k], sc[n]);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[n] = mfma32(__uint_as_float(f[e]), __uint_as_float(qf[k][e]), sc[n]);
                }
            }
        };
        auto key_of = [&](int n, int i) { return 32 * n + 8 * (i >> 2) + 4 * h + (i & 3); };
        auto mask = [&](int32_t t0, uint32_t gm) {
#pragma unroll
            for (int n = 0; n < F::NK; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int32_t t = t0 + key_of(n, i);
                    if (t < mylo || t >= myhi || t < lo || t >= hi || !(gm >> (2 * n + (i >> 3)) & 1u)) sc[n][i] = -INFINITY;
                }
        };
        auto soften = [&]() {
            float mt = sc[0][0];
#pragma unroll
            for (int n = 0; n < F::NK; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) mt = fmaxf(mt, sc[n][i]);
            mt = fmaxf(m, xmax32(mt));
            const float mu = mt == -INFINITY ? 0.f : mt;   // nothing seen yet: every weight is 0
            const float alpha = __builtin_amdgcn_exp2f((m - mu) * a.c);
            const float off = -mu * a.c;
            m = mt;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < F::NK; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[n][i] = __builtin_amdgcn_exp2f(fmaf(sc[n][i], a.c, off));
                    sum += sc[n][i];
                }
            l = fmaf(l, alpha, sum);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
        };
        // V^T fragment of keys 32 n + 16 mm + 8 e + 4 h + 0..3, dims 32 dt + l32 (bf16)
        const int i16 = lane & 15, dh = (lane >> 4) & 1;
        auto vfrag = [&](const uint8_t* vt, int r0, int e, int dt) {
            const int row = r0 + 8 * e + 4 * h + (i16 >> 2);
            const int place = (4 * dt + 2 * dh + ((i16 >> 1) & 1)) ^ (((i16 >> 2) << 2) | (2 * e + h));
            const pa_s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) pa_s16x4*)(vt + row * F::ROWB + place * 16 + (i16 & 1) * 8));
            return __builtin_bit_cast(uint2, v);
        };
        auto vfrag32 = [&](const uint8_t* vt, int row, int dt) {    // fp32: key `row` + 4 h, dim 32 dt + l32
            const int rw = row + 4 * h;
            const int f = ((rw & 3) << 2) | ((rw >> 2) & 3);
            return *reinterpret_cast<const float*>(vt + rw * F::ROWB + ((8 * dt + (l32 >> 2)) ^ f) * 16 + (l32 & 3) * 4);
        };
        auto values = [&](const uint8_t* vt) {
#pragma unroll
            for (int n = 0; n < F::NK; ++n) {
                if constexpr (F::BF) {
#pragma unroll
                    for (int mm = 0; mm < 2; ++mm) {
                        u32x4 p;
#pragma unroll
                        for (int k = 0; k < 4; ++k) p[k] = cvt_bf16x2(sc[n][8 * mm + 2 * k], sc[n][8 * mm + 2 * k + 1]);
#pragma unroll
                        for (int dt = 0; dt < 4; ++dt) {
                            const uint2 v0 = vfrag(vt, 32 * n + 16 * mm, 0, dt), v1 = vfrag(vt, 32 * n + 16 * mm, 1, dt);
                            acc[dt] = mfma32(u32x4{v0.x, v0.y, v1.x, v1.y}, p, acc[dt]);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
#pragma unroll
                        for (int dt = 0; dt < 4; ++dt)
                            acc[dt] = mfma32(vfrag32(vt, 32 * n + 8 * (i >> 2) + (i & 3), dt), sc[n][i], acc[dt]);
                }
            }
        };
        // A masked tile whose values hold infinities or NaN: 0 x inf is not 0, so a row must not meet
        // the values of keys that it does not see.  One key at a time, kept by the rows that see it.
        auto odd_values = [&](const uint8_t* vt) {
            uint32_t odd = 0;
            for (int i = lane; i < F::KB / 16; i += 64) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(vt + 16 * i);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    odd |= F::BF ? ((w[k] & 0x7F807F80u) + 0x00800080u) & 0x80008000u
                                 : ((w[k] & 0x7F800000u) + 0x00800000u) & 0x80000000u;
            }
            return __ballot(odd != 0) != 0;
        };
        auto values_by_key = [&](const uint8_t* vt, int32_t t0, uint32_t gm) {
#pragma unroll
            for (int n = 0; n < F::NK; ++n)
#pragma unroll
                for (int mm = 0; mm < 2; ++mm) {
                    u32x4 p = {0, 0, 0, 0};
                    if constexpr (F::BF)
#pragma unroll
                        for (int k = 0; k < 4; ++k) p[k] = cvt_bf16x2(sc[n][8 * mm + 2 * k], sc[n][8 * mm + 2 * k + 1]);
                    for (int kk = 0; kk < 16; ++kk) {      // key 32 n + 16 mm + kk: lanes of half (kk / 4) % 2
                        const int32_t t = t0 + 32 * n + 16 * mm + kk;
                        const bool sees = t >= mylo && t < myhi && t >= lo && t < hi && (gm >> (2 * n + mm) & 1u);
                        const bool mine = ((kk >> 2) & 1) == h;
                        const int slot = 4 * (kk >> 3) + (kk & 3);
                        float pf = 0.f;
                        u32x4 keep;
                        if constexpr (F::BF) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                keep[k] = mine && (slot >> 1) == k ? (slot & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (i == slot) pf = mine ? sc[n][8 * mm + i] : 0.f;
                        }
#pragma unroll
                        for (int dt = 0; dt < 4; ++dt) {
                            f32x16 with;
                            if constexpr (F::BF) {
                                const uint2 v0 = vfrag(vt, 32 * n + 16 * mm, 0, dt), v1 = vfrag(vt, 32 * n + 16 * mm, 1, dt);
                                with = mfma32(u32x4{v0.x, v0.y, v1.x, v1.y} & keep, p & keep, acc[dt]);
                            } else {
                                const float v = vfrag32(vt, 32 * n + 16 * mm + 8 * (kk >> 3) + (kk & 3), dt);
                                with = mfma32(mine ? v : 0.f, pf, acc[dt]);
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[dt][i] = sees ? with[i] : acc[dt][i];
                        }
                    }
                }
        };
        auto needs_mask = [&](int32_t t0, uint32_t gm) {
            return t0 < lastlo || t0 < lo || t0 + F::KT > firsthi || t0 + F::KT > hi || gm != (1u << NG) - 1;
        };
        auto tile_values = [&](const uint8_t* vt, int32_t t0, uint32_t gm, bool masked) {
            if (masked && odd_values(vt)) values_by_key(vt, t0, gm);
            else values(vt);
        };

        if constexpr (!KEYS) {
            if (lo < hi) {
                fetch_pages(t_first);
                bring(kbase, t_first, ring0);
                bring(vbase, t_first, ring0 + F::KB);
                uint32_t gm_in = gm_next;                  // of the tile that has been brought last
                fetch_pages(t_first + F::KT);
                int st = 0;
                for (int32_t t0 = t_first; t0 < hi; t0 += F::KT) {
                    const uint32_t gm = gm_in;
                    uint8_t* kt = smem + st * 2 * F::KB;
                    wait_loads<0>();
                    clear_tail(t0, kt + F::KB);
                    __syncthreads();                       // the tile is whole; the other stage is free
                    st ^= 1;
                    if (t0 + F::KT < hi) {
                        bring(kbase, t0 + F::KT, ring0 + st * 2 * F::KB);
                        bring(vbase, t0 + F::KT, ring0 + st * 2 * F::KB + F::KB);
                        gm_in = gm_next;
                        fetch_pages(t0 + 2 * F::KT);
                    }
                    if (t0 >= lasthi || t0 + F::KT <= firstlo) continue;    // no row of this wave sees the tile
                    scores(kt);
                    const bool masked = needs_mask(t0, gm);
                    if (masked) mask(t0, gm);
                    soften();
                    tile_values(kt + F::KB, t0, gm, masked);
                }
            }
            __syncthreads();
        } else {
            constexpr int L = 4 * F::CH;                   // loads of a K (or V) tile
            int32_t t0 = t_first + wave * F::KT;
            uint32_t gm_in = 0;
            if (t0 < hi) {
                fetch_pages(t0);
                bring(kbase, t0, ring0);
                bring(vbase, t0, ring0 + F::KB);
                gm_in = gm_next;
                fetch_pages(t0 + step);
            }
            for (int st = 0; t0 < hi; t0 += step) {
                const uint32_t gm = gm_in;
                uint8_t* kt = ring + st * 2 * F::KB;
                const bool more = t0 + step < hi;
                const int32_t tn = t0 + step;
                const bool masked = needs_mask(t0, gm);
                if constexpr (F::NST == 2) {
                    st ^= 1;
                    const uint32_t next = ring0 + st * 2 * F::KB;
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the other stage has been read
                    if (more) {
                        bring(kbase, tn, next);
                        bring(vbase, tn, next + F::KB);
                        gm_in = gm_next;
                        fetch_pages(tn + step);
                        wait_loads<3 * L>();
                    } else wait_loads<L>();
                    scores(kt);
                    if (masked) mask(t0, gm);
                    soften();
                    if (more) wait_loads<2 * L>();
                    else wait_loads<0>();
                } else {
                    wait_loads<L>();
                    scores(kt);
                    if (masked) mask(t0, gm);
                    soften();
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // K has been read
                    if (more) {
                        bring(kbase, tn, ring0);
                        wait_loads<L>();
                    } else wait_loads<0>();
                }
                clear_tail(t0, kt + F::KB);
                tile_values(kt + F::KB, t0, gm, masked);
                if constexpr (F::NST == 1) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // V has been read
                    if (more) {
                        bring(vbase, tn, ring0 + F::KB);
                        gm_in = gm_next;
                        fetch_pages(tn + step);
                    }
                }
            }
        }
        l = xsum32(l);

        const int64_t rec_row = idx * F::BM;               // this piece's record rows
        const bool split = u.np > 1;
        if (split && idx >= a.rec_pieces) continue;        // starts that overlap: no room for their pieces (uniform)
        float* rec_ml = a.rec + a.rec_pieces * F::BM * D;
        if constexpr (!KEYS) {
            if (live) {
                if (split) {
                    float* dst = a.rec + (rec_row + wrow0 - row0 + l32) * D;
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            *reinterpret_cast<f32x4*>(dst + 32 * dt + 2 * i + 4 * h) =
                                f32x4{acc[dt][i], acc[dt][i + 1], acc[dt][i + 2], acc[dt][i + 3]};
                    if (h == 0) *reinterpret_cast<float2*>(rec_ml + (rec_row + wrow0 - row0 + l32) * 2) = float2{m, l};
                } else {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    ET* dst = (ET*)a.out + (int64_t)(r.q0 + tok) * a.out_stride + (int64_t)(g * Hg + myrow % Hg) * D;
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float o0 = acc[dt][i] * inv, o1 = acc[dt][i + 1] * inv, o2 = acc[dt][i + 2] * inv,
                                        o3 = acc[dt][i + 3] * inv;
                            if constexpr (F::BF)
                                *reinterpret_cast<uint2*>(dst + 32 * dt + 2 * i + 4 * h) = uint2{cvt_bf16x2(o0, o1), cvt_bf16x2(o2, o3)};
                            else
                                *reinterpret_cast<f32x4*>(dst + 32 * dt + 2 * i + 4 * h) = f32x4{o0, o1, o2, o3};
                        }
                }
            }
        } else {
            __syncthreads();                               // every wave is done with its ring
            float* js = (float*)smem;                      // [4][32][132] sums
            float* jm = js + 4 * 32 * 132;                 // [4][32][2]
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f32x4*>(js + (wave * 32 + l32) * 132 + 32 * dt + 2 * i + 4 * h) =
                        f32x4{acc[dt][i], acc[dt][i + 1], acc[dt][i + 2], acc[dt][i + 3]};
            if (h == 0) *reinterpret_cast<float2*>(jm + (wave * 32 + l32) * 2) = float2{m, l};
            __syncthreads();
            const int row = threadIdx.x >> 3, d0 = 16 * (threadIdx.x & 7);
            if (row < rows) {
                float mw[4], lw[4], M = -INFINITY, L = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float2 v = *reinterpret_cast<const float2*>(jm + (w * 32 + row) * 2);
                    mw[w] = v.x;
                    lw[w] = v.y;
                    M = fmaxf(M, v.x);
                }
                const float mu = M == -INFINITY ? 0.f : M;
                float o[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float wt = __builtin_amdgcn_exp2f((mw[w] - mu) * a.c);
                    L = fmaf(wt, lw[w], L);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f32x4 v = *reinterpret_cast<const f32x4*>(js + (w * 32 + row) * 132 + d0 + i);
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[i + k] = fmaf(wt, v[k], o[i + k]);
                    }
                }
                if (split) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<f32x4*>(a.rec + (rec_row + row) * D + d0 + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
                    if (d0 == 0) *reinterpret_cast<float2*>(rec_ml + (rec_row + row) * 2) = float2{M, L};
                } else {
                    const float inv = L == 0.f ? 0.f : 1.f / L;
                    const int32_t rr = row0 + row;
                    ET* dst = (ET*)a.out + (int64_t)(r.q0 + rr / Hg) * a.out_stride + (int64_t)(g * Hg + rr % Hg) * D + d0;
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        if constexpr (F::BF)
                            *reinterpret_cast<uint2*>(dst + i) = uint2{cvt_bf16x2(o[i] * inv, o[i + 1] * inv), cvt_bf16x2(o[i + 2] * inv, o[i + 3] * inv)};
                        else
                            *reinterpret_cast<f32x4*>(dst + i) = f32x4{o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv};
                }
            }
            __syncthreads();                               // the rings are free again
        }
    }
}

// Joins the pieces of split sequences: one workgroup per (token, head) row, its waves taking every
// fourth piece.
template <typename ET>
__global__ __launch_bounds__(256) void paged_join_kernel(AttnArgs a, int BM) {
    __shared__ float so[4][D];
    __shared__ float sml[4][2];
    const Cut cut = wave_cut(a, BM);
    if (cut.L > a.cap) return;                             // nothing was split
    const int wave = first_lane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int H = a.G * a.Hg;
    const float* rec_ml = a.rec + a.rec_pieces * BM * D;
    for (int64_t w = blockIdx.x; w < (int64_t)a.T * H; w += gridDim.x) {
        const int32_t i = (int32_t)(w / H), hd = (int32_t)(w % H);
        const int s = find_seq(a.q_start, a.S, i);
        Unit u;
        if (s < 0 || !scan_units(a, cut, BM, u, [&](int k, int64_t) { return k == s; })) continue;
        if (u.np <= 1 || i < u.r.q0 || i >= u.r.q0 + u.r.qlen) continue;
        const int g = hd / a.Hg;
        const int32_t row = (int32_t)((i - u.r.q0) * a.Hg + hd % a.Hg);
        const int64_t tile = seq_tiles(u.r, a.Hg, BM) - 1 - row / BM;
        const int64_t p0 = u.base + tile * u.np * a.G + g;     // piece p is number p0 + p G
        if (p0 + (int64_t)(u.np - 1) * a.G >= a.rec_pieces) continue;
        float M = -INFINITY;
        for (int p = lane; p < u.np; p += 64) M = fmaxf(M, rec_ml[((p0 + (int64_t)p * a.G) * BM + row % BM) * 2]);
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) M = fmaxf(M, __shfl_xor(M, x, WAVE));
        const float mu = M == -INFINITY ? 0.f : M;
        float o0 = 0.f, o1 = 0.f, L = 0.f;
        for (int p = wave; p < u.np; p += 4) {
            const int64_t rr = (p0 + (int64_t)p * a.G) * BM + row % BM;
            const float2 ml = *reinterpret_cast<const float2*>(rec_ml + rr * 2);
            const float2 v = *reinterpret_cast<const float2*>(a.rec + rr * D + 2 * lane);
            const float wt = __builtin_amdgcn_exp2f((ml.x - mu) * a.c);
            L = fmaf(wt, ml.y, L);
            o0 = fmaf(wt, v.x, o0);
            o1 = fmaf(wt, v.y, o1);
        }
        __syncthreads();
        so[wave][2 * lane] = o0;
        so[wave][2 * lane + 1] = o1;
        if (lane == 0) sml[wave][0] = L;
        __syncthreads();
        if (threadIdx.x < 64) {
            L = (sml[0][0] + sml[1][0]) + (sml[2][0] + sml[3][0]);
            const float inv = L == 0.f ? 0.f : 1.f / L;
            o0 = (so[0][2 * lane] + so[1][2 * lane]) + (so[2][2 * lane] + so[3][2 * lane]);
            o1 = (so[0][2 * lane + 1] + so[1][2 * lane + 1]) + (so[2][2 * lane + 1] + so[3][2 * lane + 1]);
            ET* dst = (ET*)a.out + (int64_t)i * a.out_stride + (int64_t)hd * D + 2 * lane;
            if constexpr (sizeof(ET) == 2) *reinterpret_cast<uint32_t*>(dst) = cvt_bf16x2(o0 * inv, o1 * inv);
            else *reinterpret_cast<float2*>(dst) = float2{o0 * inv, o1 * inv};
        }
    }
}

// ---- host ------------------------------------------------------------------------------------
namespace {

constexpr int SLOTS_ROWS = 512;    // workgroups of the rows form that the card holds (2 per CU)
constexpr int SLOTS_KEYS = 256;    // of the keys form (1 per CU)
constexpr int LMIN = 512;          // shortest piece, in tokens

struct Choice { bool keys; int BM, target; int64_t pieces; };
Choice choose(int64_t T, int S, int G, int Hg, int64_t cap) {
    Choice c;
    c.keys = T * Hg <= 32 * (int64_t)S;
    c.BM = c.keys ? 32 : 128;
    c.target = c.keys ? SLOTS_KEYS : SLOTS_ROWS;
    c.pieces = max_pieces(T, S, G, Hg, c.BM, c.target, cap, LMIN);
    return c;
}
// pieces of split calls: a call is split only while its units are fewer than the target
int64_t record_pieces(const Choice& c) { return c.pieces < 2 * c.target ? c.pieces : 2 * c.target; }

template <typename ET, bool KEYS>
hipError_t launch(const AttnArgs& a, const Choice& c, hipStream_t st) {
    typedef Form<ET, KEYS> F;
    static_assert(F::BM == (KEYS ? 32 : 128), "choose()");
    const void* fn = (const void*)paged_attn_kernel<ET, KEYS>;
    hipError_t e = ensure_lds_limit(fn, F::LDS);
    if (e != hipSuccess) return e;
    const int64_t most = KEYS ? c.target : c.pieces;
    const unsigned grid = (unsigned)(c.pieces < most ? c.pieces : most);
    paged_attn_kernel<ET, KEYS><<<grid, 256, F::LDS, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t rows = (int64_t)a.T * a.G * a.Hg;
    paged_join_kernel<ET><<<(unsigned)(rows < 2048 ? rows : 2048), 256, 0, st>>>(a, F::BM);
    return hipGetLastError();
}

}  // namespace

size_t paged_attn_ws_bytes(int64_t T, int S, int G, int H, int64_t cap) {
    const Choice c = choose(T, S, G, H / G, cap);
    return (size_t)record_pieces(c) * c.BM * (D + 2) * 4;
}

hipError_t launch_paged_attn(const varrate_pages& pg, const varrate_batch& b, const void* q, int64_t q_stride, int H,
                             int causal, int window, float scale, void* out, int64_t out_stride, void* ws, hipStream_t st) {
    AttnArgs a;
    a.q = q;
    a.out = out;
    a.k = pg.k;
    a.v = pg.v;
    a.table = b.table;
    a.kv_len = b.kv_len;
    a.q_start = b.q_start;
    a.rec = (float*)ws;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.table_stride = b.table_stride;
    a.T = (int32_t)b.T;
    a.S = b.S;
    a.cap = b.width * pg.page;
    a.n_pages = (int32_t)pg.n_pages;
    a.G = pg.G;
    a.Hg = H / pg.G;
    a.shift = __builtin_ctz((unsigned)pg.page);
    a.causal = causal;
    a.window = window;
    a.lmin = LMIN;
    a.c = scale * 1.4426950408889634f;
    const Choice c = choose(b.T, b.S, pg.G, a.Hg, a.cap);
    a.target = c.target;
    a.rec_pieces = record_pieces(c);
    if (pg.dtype == VARRATE_BF16) return c.keys ? launch<uint16_t, true>(a, c, st) : launch<uint16_t, false>(a, c, st);
    return c.keys ? launch<float, true>(a, c, st) : launch<float, false>(a, c, st);
}

}  // namespace vr
