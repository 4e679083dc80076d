// Row operators of the cache of e4m3 codes, gfx950: appending key and value rows to its pages, gathering a sequence's rows
// out of them, and evicting the tokens that attention pays least.  Memory bounds them for many rows and latency for few.
//
// A block (32 tokens of one head, keys or values) has one power of two, so it belongs to one wave: 16 lanes a row, 8 values a
// lane, 4 rows at a time.
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

// Rows i .. i + n - 1, the new ones of a block of sequence s from position t on.
template <typename ET>
__device__ __forceinline__ void append_block(const Append8& p, int which, int g, int s, int32_t i, int32_t t, int32_t n) {
    const int lane = threadIdx.x & 63, rr = lane >> 4, c = 8 * (lane & 15);
    const int32_t pg = good_page(p.table[s * p.table_stride + (t >> p.pool.shift)], p.pool.n_pages);
    if (pg < 0) return;
    const int32_t slot = p.pool.slot(t), held = slot & (BLOCK - 1);
    uint8_t* scale = p.pool.scale[which] + p.pool.block(pg, g, slot);
    uint8_t* dst = p.pool.code[which] + p.pool.row(pg, g, slot) + c;
    const ET* src = (const ET*)p.x[which] + (int64_t)i * p.stride[which] + (int64_t)g * D + c;
    int was = E_LO;
    if (held) was = exponent_of(*scale);
    float x[8][8];
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (4 * k >= n) break;
        const int row = 4 * k + rr < n ? 4 * k + rr : n - 1;
        read8(src + row * p.stride[which], x[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = magnitude(x[k][e]);
            most = u > most ? u : most;
        }
    }
    int now = exponent_for(wave_most(most));
    if (held && was >= now) now = was;
    else if (held) {                                       // the rows before are rounded to the larger scale
        uint8_t* old = dst - (int64_t)held * D;
        const float back = power(was - now < -126 ? -126 : was - now);     // (2^-126 takes every code to 0 as well)
#pragma unroll 1
        for (int row = rr; row < held; row += 4) {
            float y[8];
            values8(*reinterpret_cast<const uint2*>(old + (int64_t)row * D), 1.f, y);
            *reinterpret_cast<uint2*>(old + (int64_t)row * D) = encode8(y, back);
        }
    }
    const float to = power(-now);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (4 * k >= n) break;
        if (4 * k + rr < n) *reinterpret_cast<uint2*>(dst + (int64_t)(4 * k + rr) * D) = encode8(x[k], to);
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
// 8 values of a key row and of a value row a thread and step, in the order of the output.
template <typename ET>
__global__ __launch_bounds__(256) void gather8_kernel(Pool8 pool, const int32_t* __restrict__ table, int64_t n, ET* __restrict__ K,
                                                      ET* __restrict__ V) {
    const int64_t total = n * pool.G * 16;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i >> 4;
        const int g = (int)(row % pool.G);
        const int32_t t = (int32_t)(row / pool.G), slot = pool.slot(t);
        const int32_t pg = good_page(table[t >> pool.shift], pool.n_pages);
        float k[8] = {}, v[8] = {};
        if (pg >= 0) {
            const int64_t at = pool.row(pg, g, slot) + 8 * (i & 15), b = pool.block(pg, g, slot);
            const uint2 kw = *reinterpret_cast<const uint2*>(pool.code[0] + at), vw = *reinterpret_cast<const uint2*>(pool.code[1] + at);
            values8(kw, __uint_as_float((uint32_t)pool.scale[0][b] << 23), k);
            values8(vw, __uint_as_float((uint32_t)pool.scale[1][b] << 23), v);
        }
        write8(K + i * 8, k);
        write8(V + i * 8, v);
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
};
// tokens of sequence s, those of them that have a mass
__device__ __forceinline__ int32_t tokens_of(const Evict8& p, int s) { return clamp_i32(p.kv_len[s], 0, p.cap); }

// Masses as numbers whose order is theirs: NaN before all others, both zeros alike.
__device__ __forceinline__ uint32_t rank_of(float x) {
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int SEL = 1024;                                  // threads of a selection

// Exclusive prefix sums over the workgroup of two counts below 2^16, packed; total: of all.
__device__ __forceinline__ uint32_t scan_pair(uint32_t v, uint32_t* sums, uint32_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t up = v;
#pragma unroll
    for (int m = 1; m < WAVE; m <<= 1) {
        const uint32_t y = __shfl_up(up, m, WAVE);
        if (lane >= m) up += y;
    }
    __syncthreads();                                       // the sums of the scan before have been read
    if (lane == WAVE - 1) sums[wave] = up;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < SEL / WAVE; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    return before + up - v;
}

// One workgroup a (sequence, head): the mass of the last token that stays, by its digits from the top (of 11, 11 and 10 bits),
// then the tokens above it and the first of those equal to it, in order.
__global__ __launch_bounds__(SEL) void evict8_select(Evict8 p) {
    __shared__ uint32_t hist[2048], sums[SEL / WAVE], found[2];
    const int s = (int)(blockIdx.x / (uint32_t)p.pool.G), g = (int)(blockIdx.x % (uint32_t)p.pool.G), tid = threadIdx.x;
    const int32_t n = tokens_of(p, s), m = n < p.keep ? n : p.keep;
    const float* mass = p.mass + ((int64_t)s * p.pool.G + g) * p.L;
    int32_t* index = p.index + ((int64_t)s * p.pool.G + g) * p.keep;
    float* mass_out = p.mass_out + ((int64_t)s * p.pool.G + g) * p.keep;
    if (g == 0 && tid == 0) p.len_out[s] = m;
    for (int32_t i = m + tid; i < p.keep; i += SEL) {
        index[i] = -1;
        mass_out[i] = 0.f;
    }
    // tokens [lo, hi) compete for `need` places
    const int32_t lo = p.first < n ? p.first : n, hi = n - p.recent > lo ? n - p.recent : lo;
    uint32_t need = (uint32_t)(m - lo - (n - hi)), prefix = 0;
    if (m == n) need = (uint32_t)(hi - lo);
    const bool all = need == (uint32_t)(hi - lo), none = need == 0;
    if (!all && !none) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < 2048; i += SEL) hist[i] = 0;
            __syncthreads();
            for (int32_t t = lo + tid; t < hi; t += SEL) {
                const uint32_t r = rank_of(mass[t]);
                if (pass == 0 || r >> (shift + bits) == prefix >> (shift + bits)) atomicAdd(&hist[r >> shift & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // the digit at which the count from the top reaches `need`: two digits a thread, from the top
            const int top = (1 << bits) - 1 - 2 * tid;
            const uint32_t a = top >= 0 ? hist[top] : 0, b = top >= 1 ? hist[top - 1] : 0;
            uint32_t up = a + b;
            const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
            for (int k = 1; k < WAVE; k <<= 1) {
                const uint32_t y = __shfl_up(up, k, WAVE);
                if (lane >= k) up += y;
            }
            if (lane == WAVE - 1) sums[wave] = up;
            __syncthreads();
            for (int w = 0; w < wave; ++w) up += sums[w];
            const uint32_t before = up - a - b;
            if (before < need && up >= need) {             // one thread
                const bool second = before + a < need;
                found[0] = (uint32_t)(top - (second ? 1 : 0));
                found[1] = need - before - (second ? a : 0);
            }
            __syncthreads();
            prefix |= found[0] << shift;
            need = found[1];
            __syncthreads();
        }
    }
    // ranks above `prefix`, and the first `need` equal to it
    int32_t place = 0;
    uint32_t equal = 0;
    constexpr int PER = 4;
    for (int32_t t0 = 0; t0 < n; t0 += SEL * PER) {
        uint32_t mine = 0;
        int kind[PER];                                     // 0: goes, 1: stays, 2: equal
        float x[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int32_t t = t0 + PER * tid + k;
            kind[k] = 0;
            x[k] = 0.f;
            if (t < n) {
                x[k] = mass[t];
                const uint32_t r = rank_of(x[k]);
                kind[k] = t < lo || t >= hi || all ? 1 : none ? 0 : r > prefix ? 1 : r == prefix ? 2 : 0;
            }
            mine += kind[k] == 1 ? 1u << 16 : kind[k] == 2 ? 1u : 0u;
        }
        uint32_t total, at = scan_pair(mine, sums, total);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t eq = equal + (at & 0xFFFFu);
            const int32_t to = place + (int32_t)(at >> 16) + (int32_t)((eq < need ? eq : need) - (equal < need ? equal : need));
            if (kind[k] == 1 || (kind[k] == 2 && eq < need)) {
                index[to] = t0 + PER * tid + k;
                mass_out[to] = x[k];
            }
            at += kind[k] == 1 ? 1u << 16 : kind[k] == 2 ? 1u : 0u;
        }
        const uint32_t eq = equal + (total & 0xFFFFu);
        place += (int32_t)(total >> 16) + (int32_t)((eq < need ? eq : need) - (equal < need ? equal : need));
        equal = eq;
    }
}

// A wave moves a block's rows: 32 of the tokens that stay, of one head, keys or values.
__global__ __launch_bounds__(256) void evict8_move(Evict8 p) {
    const int lane = threadIdx.x & 63, rr = lane >> 4, c = 8 * (lane & 15), G = p.pool.G;
    const int32_t blocks = (p.keep + BLOCK - 1) / BLOCK;
    const int64_t all = (int64_t)p.S * G * 2 * blocks, step = (int64_t)gridDim.x * 4;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < all; u += step) {
        const int which = (int)(u & 1), b = (int)((u >> 1) % blocks), sg = (int)((u >> 1) / blocks), s = sg / G, g = sg % G;
        const int32_t n = tokens_of(p, s), m = n < p.keep ? n : p.keep, i0 = b * BLOCK;
        if (i0 >= m) continue;
        const int32_t rows = m - i0 < BLOCK ? m - i0 : BLOCK;
        const int32_t to = good_page(p.into[s * p.into_stride + (i0 >> p.pool.shift)], p.pool.n_pages);
        if (to < 0) continue;
        // lane l knows row l
        int64_t from = -1;
        float scale = 0.f;
        if (lane < rows) {
            const int32_t t = p.index[(int64_t)sg * p.keep + i0 + lane];
            const int32_t pg = t >= 0 && t < n ? good_page(p.table[s * p.table_stride + (t >> p.pool.shift)], p.pool.n_pages) : -1;
            if (pg >= 0) {
                from = p.pool.row(pg, g, p.pool.slot(t));
                scale = __uint_as_float((uint32_t)p.pool.scale[which][p.pool.block(pg, g, p.pool.slot(t))] << 23);
            }
        }
        float x[8][8];
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int row = 4 * k + rr;
            const int64_t at = __shfl(from, row, WAVE);
            const float sc = __shfl(scale, row, WAVE);
            uint2 w = {0, 0};
            if (at >= 0) w = *reinterpret_cast<const uint2*>(p.pool.code[which] + at + c);
            values8(w, sc, x[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t v = magnitude(x[k][e]);
                most = v > most ? v : most;
            }
        }
        const int now = exponent_for(wave_most(most));
        const float s_to = power(-now);
        const int32_t slot = p.pool.slot(i0);
        uint8_t* dst = p.pool.code[which] + p.pool.row(to, g, slot) + c;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (4 * k + rr < rows) *reinterpret_cast<uint2*>(dst + (int64_t)(4 * k + rr) * D) = encode8(x[k], s_to);
        if (lane == 0) p.pool.scale[which][p.pool.block(to, g, slot)] = (uint8_t)(now + 127);
    }
}

unsigned grid_of(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

template <typename ET>
hipError_t append_as(const Append8& p, hipStream_t st) {
    const int64_t rows = (int64_t)p.T * 2 * p.pool.G;
    // few rows: one a wave, so that single tokens spread over the card
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
    const unsigned grid = grid_of((n * pg.G * 16 + 255) / 256, 16384);
    if (dtype == VARRATE_BF16) gather8_kernel<uint16_t><<<grid, 256, 0, st>>>(pool_of(pg), table, n, (uint16_t*)K, (uint16_t*)V);
    else gather8_kernel<float><<<grid, 256, 0, st>>>(pool_of(pg), table, n, (float*)K, (float*)V);
    return hipGetLastError();
}

hipError_t launch_paged8_evict(const varrate_pages8& pg, const Evict8Args& e, hipStream_t st) {
    const int64_t cap = (int64_t)e.width * pg.page;
    const Evict8 p = {pool_of(pg), e.table, e.into, e.kv_len, e.table_stride, e.into_stride, e.mass, e.index, e.mass_out, e.len_out,
                      e.L, e.S, (int32_t)(cap < e.L ? cap : e.L), (int32_t)e.keep, (int32_t)e.first, (int32_t)e.recent};
    evict8_select<<<(unsigned)e.S * (unsigned)pg.G, SEL, 0, st>>>(p);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const int64_t waves = (int64_t)e.S * pg.G * 2 * ((e.keep + BLOCK - 1) / BLOCK);
    evict8_move<<<grid_of((waves + 3) / 4, 1 << 20), 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vr
