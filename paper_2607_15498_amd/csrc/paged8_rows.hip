// Row operators of the cache of e4m3 codes, gfx950: appending key and value rows to its pages, gathering a sequence's rows
// out of them, and evicting the tokens that attention pays least.  Memory bounds append and gather for many rows (32768 tokens of 8
// heads, bf16: 40 us, 5.1 TB/s, and 30 us, 6.7 TB/s) and latency for few (64 single tokens: 5 us).
//
// A block (32 tokens of one head, keys or values) has one power of two, so it belongs to one wave: 16 lanes a row, 8 values a
// lane, 4 rows at a time.
#include <type_traits>

#include "vr_codes.h"
#include "vr_pages.h"

namespace vr {
namespace {

struct Pool8 {
    uint8_t *code[2], *scale[2];     // of keys, of values
    int32_t G, n_pages, shift;
    // where row `slot` of page pg lies, and its block's scale
    __device__ __forceinline__ int64_t row(int32_t pg, int g, int32_t slot) const { return ((((int64_t)pg * G + g) << shift) + slot) * D; }
    __device__ __forceinline__ int64_t block(int32_t pg, int g, int32_t slot) const {
        return (((int64_t)pg * G + g) << (shift - 5)) + (slot >> 5);
    }
    __device__ __forceinline__ int32_t slot(int32_t t) const { return t & ((1 << shift) - 1); }
};
Pool8 pool_of(const varrate_pages8& pg) {
    return Pool8{{(uint8_t*)pg.k, (uint8_t*)pg.v}, {(uint8_t*)pg.k_scale, (uint8_t*)pg.v_scale}, pg.G, (int32_t)pg.n_pages,
                 __builtin_ctz((unsigned)pg.page)};
}

// ---- append -------------------------------------------------------------------------------------
struct Append8 {
    Pool8 pool;
    const void* x[2];                // new rows of keys, of values
    int64_t stride[2];               // elements between tokens
    const int32_t *table, *kv_len, *q_start;
    int64_t table_stride;
    int32_t T, S, cap;
};

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// 8 values as they lie in memory, read once.
template <typename ET> struct Raw8;
template <> struct Raw8<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void read(const uint16_t* p) { w = __builtin_nontemporal_load((const u32x4*)p); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[2 * k] = bf_lo(w[k]);
            x[2 * k + 1] = bf_hi(w[k]);
        }
    }
    // the largest of their magnitudes' bits and `most`, whether numbers or not
    typedef u16x2 Most;
    __device__ __forceinline__ void raise(Most& most) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[k] & 0x7FFF7FFFu));
    }
    static __device__ __forceinline__ uint32_t bits(Most m) { return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16; }
};
template <> struct Raw8<float> {
    f32x4 w[2];
    __device__ __forceinline__ void read(const float* p) {
        w[0] = __builtin_nontemporal_load((const f32x4*)p);
        w[1] = __builtin_nontemporal_load((const f32x4*)(p + 4));
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = w[k >> 2][k & 3];
    }
    typedef uint32_t Most;
    __device__ __forceinline__ void raise(Most& most) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t u = __float_as_uint(w[k >> 2][k & 3]) & 0x7FFFFFFFu;
            most = u > most ? u : most;
        }
    }
    static __device__ __forceinline__ uint32_t bits(Most m) { return m; }
};

// Rows i .. i + n - 1, the new ones of a block of sequence s from position t on.  They are asked for before the page is looked up
// and kept as they are (32768 tokens of 8 heads, bf16: 68 us with the page first and the rows as fp32, 40 so).
template <typename ET>
__device__ __forceinline__ void append_block(const Append8& p, int which, int g, int s, int32_t i, int32_t t, int32_t n) {
    const int lane = threadIdx.x & 63, rr = lane >> 4, c = 8 * (lane & 15);
    const ET* src = (const ET*)p.x[which] + (int64_t)i * p.stride[which] + (int64_t)g * D + c;
    Raw8<ET> x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (4 * k < n) x[k].read(src + (4 * k + rr < n ? 4 * k + rr : n - 1) * p.stride[which]);
    const int32_t pg = good_page(p.table[s * p.table_stride + (t >> p.pool.shift)], p.pool.n_pages);
    if (pg < 0) return;
    const int32_t slot = p.pool.slot(t), held = slot & (BLOCK - 1);
    uint8_t* scale = p.pool.scale[which] + p.pool.block(pg, g, slot);
    uint8_t* dst = p.pool.code[which] + p.pool.row(pg, g, slot) + c;
    int was = E_LO;
    if (held) was = exponent_of(*scale);
    typename Raw8<ET>::Most top = {};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (4 * k < n) x[k].raise(top);
    uint32_t most = wave_most(Raw8<ET>::bits(top));
    if (most >= 0x7F800000u) {                             // infinities or NaN among them: of the others
        most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (4 * k < n) {
                float y[8];
                x[k].get(y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t u = magnitude(y[e]);
                    most = u > most ? u : most;
                }
            }
        most = wave_most(most);
    }
    int now = exponent_for(most);
    if (held && was >= now) now = was;
    else if (held) {                                       // the rows before are rounded to the larger scale
        uint8_t* old = dst - (int64_t)held * D;
        const float back = power(was - now < -126 ? -126 : was - now);     // (2^-126 takes every code to 0 as well)
#pragma unroll 1
        for (int row = rr; row < held; row += 4) {
            float y[8];
            values8(*reinterpret_cast<const uint2*>(old + (int64_t)row * D), 1.f, y);
            *reinterpret_cast<uint2*>(old + (int64_t)row * D) = encode8<false>(y, back);
        }
    }
    const float to = power(-now);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (4 * k + rr < n) {
            float y[8];
            x[k].get(y);
            const uint2 w = now == E_HI ? encode8<true>(y, to) : encode8<false>(y, to);
            __builtin_nontemporal_store((uint64_t)w.y << 32 | w.x, (uint64_t*)(dst + (int64_t)(4 * k + rr) * D));
        }
    if (lane == 0) *scale = (uint8_t)(now + 127);
}

// A wave has W rows of the call and one (head, keys or values): of these rows it takes the blocks whose first new row is among them.
template <typename ET, int W>
__global__ __launch_bounds__(256) void append8_kernel(Append8 p) {
    const int lane = threadIdx.x & 63, streams = 2 * p.pool.G;
    const int64_t all = ((int64_t)p.T + W - 1) / W * streams, step = (int64_t)gridDim.x * 4;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < all; u += step) {
        const int stream = (int)(u % streams), which = stream & 1, g = stream >> 1;
        const int32_t i0 = (int32_t)(u / streams) * W, i = i0 + lane % W;
        int32_t t = -1, n = 0;
        int s = -1;
        if (i < p.T && lane < W && (s = find_seq(p.q_start, p.S, i)) >= 0) {
            const SeqRange r = seq_range(p.q_start[s], p.q_start[s + 1], p.kv_len[s], p.T, p.cap);
            // a length beyond the table would move the rows: nothing is written for it
            if (p.kv_len[s] >= 0 && p.kv_len[s] <= p.cap) t = r.klen - r.qlen + (i - r.q0);
            if (t >= 0 && (i == r.q0 || (t & (BLOCK - 1)) == 0)) {
                const int32_t room = BLOCK - (t & (BLOCK - 1)), left = r.q0 + r.qlen - i;
                n = room < left ? room : left;
            }
        }
        uint64_t todo = __ballot(n > 0);
        while (todo) {
            const int l = __builtin_ctzll(todo);
            todo &= todo - 1;
            append_block<ET>(p, which, g, __builtin_amdgcn_readlane(s, l), i0 + l, __builtin_amdgcn_readlane(t, l),
                             __builtin_amdgcn_readlane(n, l));
        }
    }
}

// ---- gather -------------------------------------------------------------------------------------
// 16 bytes of a key row's and a value row's output a thread and step, non-temporal; a wave has 4 (fp32 2) tokens of one head, whose
// codes lie together.  32768 tokens of 8 heads, bf16: 34 -> 30 us (6.7 TB/s) against ordinary stores; fp32 with 32 bytes a thread
// lost by them (16384 tokens: 28 -> 51 us).
__device__ __forceinline__ u32x4 values_out(uint2 w, float s, uint16_t) {
    float x[8];
    values8(w, s, x);
    return u32x4{cvt_bf16x2(x[0], x[1]), cvt_bf16x2(x[2], x[3]), cvt_bf16x2(x[4], x[5]), cvt_bf16x2(x[6], x[7])};
}
__device__ __forceinline__ f32x4 values_out(uint32_t w, float s, float) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return f32x4{a[0] * s, a[1] * s, b[0] * s, b[1] * s};
}
template <typename ET>
__global__ __launch_bounds__(256) void gather8_kernel(Pool8 pool, const int32_t* __restrict__ table, int64_t n, ET* __restrict__ K,
                                                      ET* __restrict__ V) {
    constexpr int PER = 16 / (int)sizeof(ET), ROW = D / PER, TOKENS = 64 / ROW;
    typedef std::conditional_t<PER == 8, uint2, uint32_t> Codes;
    const int64_t total = (n + TOKENS - 1) / TOKENS * pool.G * 64;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t wave = i >> 6, t = wave / pool.G * TOKENS + (i & 63) / ROW;
        const int g = (int)(wave % pool.G), c = (int)(i % ROW) * PER;
        if (t >= n) continue;
        const int32_t slot = pool.slot((int32_t)t), pg = good_page(table[t >> pool.shift], pool.n_pages);
        Codes k = {}, v = {};
        float ks = 0.f, vs = 0.f;
        if (pg >= 0) {
            const int64_t at = pool.row(pg, g, slot) + c, b = pool.block(pg, g, slot);
            k = *reinterpret_cast<const Codes*>(pool.code[0] + at);
            v = *reinterpret_cast<const Codes*>(pool.code[1] + at);
            ks = __uint_as_float((uint32_t)pool.scale[0][b] << 23);
            vs = __uint_as_float((uint32_t)pool.scale[1][b] << 23);
        }
        const int64_t to = (t * pool.G + g) * D + c;
        const auto ko = values_out(k, ks, ET()), vo = values_out(v, vs, ET());
        __builtin_nontemporal_store(ko, (decltype(values_out(k, ks, ET()))*)(K + to));
        __builtin_nontemporal_store(vo, (decltype(values_out(v, vs, ET()))*)(V + to));
    }
}

// ---- eviction -----------------------------------------------------------------------------------
struct Evict8 {
    Pool8 pool;
    const int32_t *table, *into, *kv_len;
    int64_t table_stride, into_stride;
    const float* mass;
    int32_t* index;
    float* mass_out;
    int32_t* len_out;
    int64_t L;
    int32_t S, cap, keep, first, recent;
    uint32_t from;                   // the selection's first (sequence, head) of this launch
};
// tokens of sequence s, those of them that have a mass
__device__ __forceinline__ int32_t tokens_of(const Evict8& p, int s) { return clamp_i32(p.kv_len[s], 0, p.cap); }

// Masses as numbers whose order is theirs: both zeros alike, NaN (1) before all others; 0 is no token's, and ALWAYS is a token's
// that stays whatever its mass.
constexpr uint32_t ALWAYS = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t rank_of(float x) {
    if (x != x) return 1;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float mass_of(uint32_t rank) {
    return rank == 1 ? NAN : __uint_as_float(rank & 0x80000000u ? rank ^ 0x80000000u : ~rank);
}
__device__ __forceinline__ uint32_t count_below(uint64_t mask, uint32_t from) {    // lanes below this one, added to `from`
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, from));
}

constexpr int SEL = 1024, SEL_WAVES = SEL / WAVE;          // threads of a selection
constexpr int SEL_PART = 32768;                            // tokens whose ranks it holds at once

// The counts of the waves before this one, and of all.
__device__ __forceinline__ uint32_t waves_before(const uint32_t* sums, int wave, uint32_t& total) {
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < SEL_WAVES; w += 4) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(sums + w);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            before += w + k < wave ? v[k] : 0;
            total += v[k];
        }
    }
    return before;
}

// One workgroup a (sequence, head): the rank of the last of the m tokens that stay, by its digits from the top (of 10, 11 and 11
// bits), then the tokens above it and the first of those equal to it, in order.  Ranks lie in shared memory, a part of 32768 at a
// time (one alone is read once; of several, a pass begins with the one that is held: 65536 tokens 78 -> 64 us, both launches); a wave has 256
// that follow each other, 4 a lane.  The instructions of its CU bound it: about 20 a token and pass, 64 tokens a row and ranges
// compared, took 42 us for 32768 tokens (of one head or of 8, a CU each), these take 22: 6 to read them and count the first digit, 3
// + 1 a pass and its digit, 2 to count and 6 to place.  Rows kept in registers, every pass's loop unrolled, took 58.
__global__ __launch_bounds__(SEL) void evict8_select(Evict8 p) {
    extern __shared__ __align__(16) uint32_t ranks[];
    __shared__ __align__(16) uint32_t hist[4096];          // a digit's copies lie together: equal digits of one read fall into different ones
    __shared__ __align__(16) uint32_t sums[SEL_WAVES];
    __shared__ uint32_t found[3];                          // the digit, how many of its ranks stay, and of how many
    const uint32_t u = p.from + blockIdx.x;
    const int s = (int)(u / (uint32_t)p.pool.G), g = (int)(u % (uint32_t)p.pool.G), tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t n = tokens_of(p, s), m = n < p.keep ? n : p.keep;
    const float* mass = p.mass + ((int64_t)s * p.pool.G + g) * p.L;
    int32_t* index = p.index + ((int64_t)s * p.pool.G + g) * p.keep;
    float* mass_out = p.mass_out + ((int64_t)s * p.pool.G + g) * p.keep;
    if (g == 0 && tid == 0) p.len_out[s] = m;
    for (int32_t i = m + tid; i < p.keep; i += SEL) {
        index[i] = -1;
        mass_out[i] = 0.f;
    }
    if (m == 0) return;
    const int32_t lo = p.first, hi = n - p.recent;         // tokens before and from there on stay (first + recent <= m unless all do)
    const int parts = (n + SEL_PART - 1) / SEL_PART;
    int turns = 0, at = 0, held = -1;                      // of a part: reads a lane; the lane's first; the part that is held
    // (the first pass's counts are taken on the way)
    auto load = [&](int part, bool first) {
        const int32_t t0 = part * SEL_PART, len = n - t0 < SEL_PART ? n - t0 : SEL_PART;
        turns = (len + 4 * SEL - 1) / (4 * SEL);
        at = wave * turns * 64 + lane;
        if (part == held) return;
        if (held >= 0) __syncthreads();                    // the part before has been read
        held = part;
        for (int i0 = tid; i0 < turns * 4 * SEL; i0 += 8 * SEL) {      // 8 reads at a time (tokens that there are)
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = mass[t0 + (i0 + k * SEL < len ? i0 + k * SEL : len - 1)];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + k * SEL, t = t0 + i;
                const uint32_t u = rank_of(x[k]), r = i >= len ? 0 : t < lo || t >= hi ? ALWAYS : u;
                if (i < turns * 4 * SEL) {
                    ranks[i] = r;
                    if (first) atomicAdd(&hist[(r >> 22) * 4 + (lane & 3)], 1u);
                }
            }
        }
        __syncthreads();
    };
    const u32x4* quads = reinterpret_cast<const u32x4*>(ranks);
    uint32_t need = (uint32_t)m, prefix = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 22 : pass == 1 ? 11 : 0, bits = pass == 0 ? 10 : 11;
        reinterpret_cast<uint4*>(hist)[tid] = uint4{0, 0, 0, 0};
        __syncthreads();
#pragma unroll 1
        for (int j = 0; j < parts; ++j) {                  // up and down in turn: a pass begins with the part that is held
            load(pass & 1 ? parts - 1 - j : j, pass == 0);
            if (pass) {
                for (int i = 0; i < turns; ++i) {          // few begin as those before
                    const u32x4 r = quads[at + 64 * i];
                    bool in[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) in[k] = (r[k] ^ prefix) >> (shift + 11) == 0;
                    if (in[0] || in[1] || in[2] || in[3])
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (in[k]) atomicAdd(&hist[(r[k] >> shift & 2047u) * 2 + (lane & 1)], 1u);
                }
            }
        }
        __syncthreads();
        // the digit at which the count from the top reaches `need`: two digits a thread, from the top
        const int top = (1 << bits) - 1 - 2 * tid;
        uint32_t a = 0, b = 0;
        if (top >= 1) {
            if (pass == 0) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(hist + 4 * top), y = *reinterpret_cast<const u32x4*>(hist + 4 * (top - 1));
                a = x[0] + x[1] + x[2] + x[3];
                b = y[0] + y[1] + y[2] + y[3];
            } else {
                const u32x4 x = *reinterpret_cast<const u32x4*>(hist + 2 * (top - 1));
                a = x[2] + x[3];
                b = x[0] + x[1];
            }
        }
        uint32_t up = a + b, total;
#pragma unroll
        for (int k = 1; k < WAVE; k <<= 1) {
            const uint32_t y = __shfl_up(up, k, WAVE);
            if (lane >= k) up += y;
        }
        if (lane == WAVE - 1) sums[wave] = up;
        __syncthreads();
        up += waves_before(sums, wave, total);
        const uint32_t before = up - a - b;
        if (before < need && up >= need) {                 // one thread
            const bool second = before + a < need;
            found[0] = (uint32_t)(top - (second ? 1 : 0));
            found[1] = need - before - (second ? a : 0);
            found[2] = second ? b : a;
        }
        __syncthreads();
        prefix |= found[0] << shift;
        need = found[1];
        if (found[2] == need && prefix) {                  // all that begin so stay: no further digits
            prefix -= 1;
            need = 0;
            break;
        }
    }
    // ranks above `prefix`, and the first `need` equal to it: counted per wave (above and equal, 16 bits each), then placed, the
    // last part first
    uint32_t place = (uint32_t)m - need, equal = found[2]; // in this part and those before (`equal` counts only if need does)
#pragma unroll 1
    for (int part = parts - 1; part >= 0; --part) {
        load(part, false);
        uint32_t mine = 0;
        for (int i = 0; i < turns; ++i) {
            const u32x4 r = quads[at + 64 * i];
#pragma unroll
            for (int k = 0; k < 4; ++k) mine += (r[k] > prefix ? 1u << 16 : 0u) + (r[k] == prefix ? 1u : 0u);
        }
#pragma unroll
        for (int k = 1; k < WAVE; k <<= 1) mine += __shfl_xor(mine, k, WAVE);
        __syncthreads();                                   // the sums before have been read
        if (lane == 0) sums[wave] = mine;
        __syncthreads();
        // a part has up to 2^15 of either: 16 waves' sums do not carry
        uint32_t total;
        const uint32_t before = waves_before(sums, wave, total);
        place -= total >> 16;
        equal -= total & 0xFFFFu;
        uint32_t to0 = place + (before >> 16), eq0 = equal + (before & 0xFFFFu);
        for (int i = 0; i < turns; ++i) {
            const u32x4 r = quads[at + 64 * i];
            uint64_t above[4], same[4], any = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                above[k] = __ballot(r[k] > prefix);
                same[k] = __ballot(r[k] == prefix);
                any |= same[k];
            }
            // (byte offsets of 32 bits: keep is 2^30 at most)
            auto put = [&](int k, uint32_t slot) {
                const int32_t t = part * SEL_PART + 4 * (at + 64 * i) + k;
                *(int32_t*)((uint8_t*)index + 4 * slot) = t;
                *(float*)((uint8_t*)mass_out + 4 * slot) = r[k] == ALWAYS ? mass[t] : mass_of(r[k]);
            };
            uint32_t to = to0 + (eq0 < need ? eq0 : need);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                to = count_below(above[k], to);
                to0 += __builtin_popcountll(above[k]);
            }
            if (!any) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (r[k] > prefix) put(k, to);
                    to += r[k] > prefix ? 1 : 0;
                }
            } else {
                uint32_t eq = eq0;
                to -= eq0 < need ? eq0 : need;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    eq = count_below(same[k], eq);
                    eq0 += __builtin_popcountll(same[k]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool is = r[k] == prefix;
                    if (r[k] > prefix || (is && eq < need)) put(k, to + (eq < need ? eq : need));
                    to += r[k] > prefix ? 1 : 0;
                    eq += is ? 1 : 0;
                }
            }
        }
    }
}

// A wave moves a block's rows: 32 of the tokens that stay, of one head, keys or values.  A chain of three reads (token, page,
// row) and what its vector work takes bound it: 6554 of 32768 tokens of 8 heads 10 us (13.5 as values instead of codes).
__global__ __launch_bounds__(256) void evict8_move(Evict8 p) {
    const int lane = threadIdx.x & 63, rr = lane >> 4, c = 8 * (lane & 15), G = p.pool.G;
    const int32_t blocks = (p.keep + BLOCK - 1) / BLOCK;
    const int64_t all = (int64_t)p.S * G * 2 * blocks, step = (int64_t)gridDim.x * 4;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < all; u += step) {
        const int which = (int)(u & 1), b = (int)((u >> 1) % blocks), sg = (int)((u >> 1) / blocks), s = sg / G, g = sg % G;
        const int32_t i0 = b * BLOCK;
        const int32_t raw = p.into[s * p.into_stride + (i0 >> p.pool.shift)];
        // lane l knows row l; the rows that stay come first
        const int32_t t = lane < BLOCK && i0 + lane < p.keep ? p.index[(int64_t)sg * p.keep + i0 + lane] : -1;
        const int rows = __builtin_popcountll(__ballot(t >= 0));
        const int32_t to = good_page(raw, p.pool.n_pages);
        if (to < 0 || !rows) continue;
        int64_t from = -1;
        float scale = 0.f;
        if (t >= 0 && t < p.cap) {
            const int32_t pg = good_page(p.table[s * p.table_stride + (t >> p.pool.shift)], p.pool.n_pages);
            if (pg >= 0) {
                from = p.pool.row(pg, g, p.pool.slot(t));
                scale = __uint_as_float((uint32_t)p.pool.scale[which][p.pool.block(pg, g, p.pool.slot(t))] << 23);
            }
        }
        uint2 w[8];
        float sc[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t at = __shfl(from, 4 * k + rr, WAVE);
            sc[k] = __shfl(scale, 4 * k + rr, WAVE);
            w[k] = uint2{0, 0};
            if (at >= 0) w[k] = *reinterpret_cast<const uint2*>(p.pool.code[which] + at + c);
        }
        // the largest magnitude: codes without their signs are in the order of what they stand for (0x7F: NaN)
        uint32_t most = 0;
        bool nan = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const u16x2 m0 = __builtin_elementwise_max(__builtin_bit_cast(u16x2, w[k].x & 0x007F007Fu), __builtin_bit_cast(u16x2, w[k].x >> 8 & 0x007F007Fu));
            const u16x2 m1 = __builtin_elementwise_max(__builtin_bit_cast(u16x2, w[k].y & 0x007F007Fu), __builtin_bit_cast(u16x2, w[k].y >> 8 & 0x007F007Fu));
            const u16x2 m = __builtin_elementwise_max(m0, m1);
            const int top = m[0] > m[1] ? m[0] : m[1];
            nan = nan || top == 0x7F;
            const uint32_t v = __float_as_uint(__builtin_amdgcn_cvt_f32_fp8(top, 0) * sc[k]);
            most = v > most ? v : most;
        }
        if (__any(nan)) {
            most = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float x[8];
                values8(w[k], sc[k], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t v = magnitude(x[e]);
                    most = v > most ? v : most;
                }
            }
        }
        const int now = exponent_for(wave_most(most));
        const int32_t slot = p.pool.slot(i0);
        uint8_t* dst = p.pool.code[which] + p.pool.row(to, g, slot) + c;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (4 * k + rr < rows) {
                float x[8];
                values8(w[k], 1.f, x);
                // from the row's scale to the new one: a finite power, as 0 times infinity would be NaN.  More than 2^127 only rows of zeros
                // (and NaN) can be above their new block, and 2^-126 takes every code to 0.
                const int up = (int)(__float_as_uint(sc[k]) >> 23) - 127 - now;
                *reinterpret_cast<uint2*>(dst + (int64_t)(4 * k + rr) * D) = encode8<false>(x, power(up < -126 ? -126 : up > 127 ? 127 : up));
            }
        if (lane == 0) p.pool.scale[which][p.pool.block(to, g, slot)] = (uint8_t)(now + 127);
    }
}

unsigned grid_of(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

template <typename ET>
hipError_t append_as(const Append8& p, hipStream_t st) {
    const int64_t rows = (int64_t)p.T * 2 * p.pool.G;
    // Few rows: one a wave, so that single tokens spread over the card, as starts are on the device and a chunk could as well be many
    // sequences.  8 heads, calls one after another, us, with one and with 32 rows a wave: 64 single tokens, bf16 7.6 and 50, 1024 22 and 50
    // (fp32 7.2 and 52, 27 and 52); a prompt of 512 7.8 and 7.9 (11 and 7.4), of 1024 12 and 8 (19 and 7.3), of 2048 20 and 8 (36 and 8).
    if (rows <= 16384) append8_kernel<ET, 1><<<grid_of((rows + 3) / 4, 1 << 20), 256, 0, st>>>(p);
    else append8_kernel<ET, 32><<<grid_of((((int64_t)p.T + 31) / 32 * 2 * p.pool.G + 3) / 4, 1 << 20), 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged8_append(const varrate_pages8& pg, const varrate_batch& b, int dtype, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, hipStream_t st) {
    const Append8 p = {pool_of(pg), {k, v}, {k_stride, v_stride}, b.table, b.kv_len, b.q_start, b.table_stride, (int32_t)b.T, b.S,
                       b.width * pg.page};
    return dtype == VARRATE_BF16 ? append_as<uint16_t>(p, st) : append_as<float>(p, st);
}

hipError_t launch_paged8_gather(const varrate_pages8& pg, const int32_t* table, int64_t n, int dtype, void* K, void* V, hipStream_t st) {
    const int64_t tokens = dtype == VARRATE_BF16 ? 4 : 2;  // of a wave
    const unsigned grid = grid_of(((n + tokens - 1) / tokens * pg.G + 3) / 4, 16384);
    if (dtype == VARRATE_BF16) gather8_kernel<uint16_t><<<grid, 256, 0, st>>>(pool_of(pg), table, n, (uint16_t*)K, (uint16_t*)V);
    else gather8_kernel<float><<<grid, 256, 0, st>>>(pool_of(pg), table, n, (float*)K, (float*)V);
    return hipGetLastError();
}

hipError_t launch_paged8_evict(const varrate_pages8& pg, const Evict8Args& e, hipStream_t st) {
    const int64_t cap = (int64_t)e.width * pg.page;
    Evict8 p = {pool_of(pg), e.table, e.into, e.kv_len, e.table_stride, e.into_stride, e.mass, e.index, e.mass_out, e.len_out,
                e.L, e.S, (int32_t)(cap < e.L ? cap : e.L), (int32_t)e.keep, (int32_t)e.first, (int32_t)e.recent, 0};
    const size_t lds = 4 * (size_t)(p.cap < SEL_PART ? (p.cap + 4 * SEL - 1) / (4 * SEL) * (4 * SEL) : SEL_PART);
    hipError_t err = ensure_lds_limit((const void*)evict8_select, 4 * SEL_PART);
    if (err != hipSuccess) return err;
    // a launch has fewer than 2^32 threads: 2^21 selections (a loop in the kernel instead: 32.3 -> 32.8 us for 32768 tokens of 8 heads)
    constexpr uint32_t MOST = 1u << 21;
    const uint32_t all = (uint32_t)e.S * (uint32_t)pg.G;
    for (; p.from < all; p.from += MOST) {
        evict8_select<<<all - p.from < MOST ? all - p.from : MOST, SEL, lds, st>>>(p);
        err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    const int64_t waves = (int64_t)e.S * pg.G * 2 * ((e.keep + BLOCK - 1) / BLOCK);
    evict8_move<<<grid_of((waves + 3) / 4, 1 << 20), 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vr
