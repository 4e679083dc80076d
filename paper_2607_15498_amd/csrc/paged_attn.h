// What the paged attention's kernels share: the call's cut, a piece's addresses and masks, the products of
// 32-key blocks and the few-rows form.  The head of paged_attn.hip describes the whole.
#pragma once
#include <type_traits>

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
    float* rec;                     // partial rows [rec_rows][128], then their [rec_rows][2] (max, sum), then the shares
    int64_t q_stride, out_stride;   // elements between tokens
    int64_t table_stride;
    int64_t rec_rows, most_units;
    int32_t T, S, cap, n_pages, G, Hg, shift;
    int32_t causal, window;
    Costs costs;
    float c, c_lo;                  // softmax scale x log2 e, and what c lacks of it (fp32 layers)
};

// rows of a bad page: 1 KB of zeros
__device__ const uint4 pa_zeros[64] = {};

// The lane's number, formed where it is used: what is derived from it is not kept for a whole loop.  (A register
// that is spilt there costs more than its load: the wait for it is one for all of the stages that are under way.)
__device__ __forceinline__ int lane_now() {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
}

template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(float a, float b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
// a + both halves of a bf16 pair
__device__ __forceinline__ float add_pair(uint32_t w, float a) {
    const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), one, a, false);
}

// a value that all lanes hold, as a scalar
__device__ __forceinline__ int32_t first_lane(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t first_lane(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int32_t)(uint32_t)v);
    return (int64_t)((uint64_t)(uint32_t)first_lane((int32_t)(v >> 32)) << 32 | lo);
}

// One direct-to-LDS load: 16 bytes per lane from base + off to LDS byte address dst + 16 lane.  ONCE: non-temporal, for keys
// and values of few rows, which no other workgroup reads unless sequences share pages (one token over 131072: 113 -> 103 us;
// 32 over 100 .. 21800: 286 -> 261; but 32 over the same 4096 tokens: 54 -> 60).
template <bool ONCE = false>
__device__ __forceinline__ void lds_load(const void* base, uint32_t off, uint32_t dst) {
    const uint64_t b = (uint64_t)first_lane((int64_t)base);      // scalars, wherever the compiler keeps them
    const int32_t d = first_lane((int)dst);
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(b), "s"(d) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(b), "s"(d) : "memory", "m0");
}
__device__ __forceinline__ int64_t lane64(int64_t v, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane));
}

// ---- who does what, computed by every wave from the device lengths ------------------------------
__device__ __forceinline__ float first_lane(float v) {
    return __uint_as_float((uint32_t)first_lane((int32_t)__float_as_uint(v)));
}
__device__ __forceinline__ SeqRange load_range(const AttnArgs& a, int s) {
    SeqRange r = {0, 0, 0};
    if (s < a.S) r = seq_range(a.q_start[s], a.q_start[s + 1], a.kv_len[s], a.T, a.cap);
    return r;
}
struct Plan { int64_t head, units; Split split; };         // cost of a head's work; tiles x heads
// `first`: the first 64 sequences, kept for the searches.
__device__ __forceinline__ Plan wave_plan(const AttnArgs& a, const SeqRange& first) {
    const int lane = threadIdx.x & 63, n = a.S < 64 ? a.S : 64;
    Sums s;
    for (int s0 = 0; s0 < a.S; s0 += 64)
        sum_up(s, s0 ? load_range(a, s0 + lane) : first, a.G, a.Hg, a.causal, a.window, a.costs);
    for (int m = 1; m < n; m <<= 1) {
        s.head += (uint64_t)__shfl_xor((int64_t)s.head, m, WAVE);
        s.units += __shfl_xor(s.units, m, WAVE);
        s.total += __shfl_xor(s.total, m, WAVE);
        s.many += __shfl_xor(s.many, m, WAVE);
        s.units_many += __shfl_xor(s.units_many, m, WAVE);
        s.longest = fmaxf(s.longest, __shfl_xor(s.longest, m, WAVE));
    }
    const int64_t head = first_lane((int64_t)s.head);
    s.units = units_of(first_lane(s.units), a.most_units);
    s.total = first_lane(s.total);
    s.many = first_lane(s.many);
    s.units_many = first_lane(s.units_many);
    s.longest = first_lane(s.longest);
    if (!a.rec_rows || !s.units) return Plan{head, s.units, Split{0, 0}};
    const Split p = split_of(s, (int)gridDim.x, a.costs);
    return Plan{head, s.units, Split{first_lane(p.among), first_lane(p.same)}};
}
// The sequence into whose measure number x falls.  at, before: the 64 sequences that it was found among and the measure
// before them: a search for a number behind goes on from there.
struct Search { int32_t at = 0; int64_t before = 0; };
struct Found { SeqRange r; int32_t s; int64_t base; };
template <typename M>
__device__ __forceinline__ bool find(const AttnArgs& a, const SeqRange& first, int64_t x, Search& from, Found& f, M&& measure) {
    const int lane = threadIdx.x & 63, lanes = a.S < 64 ? a.S : 64;
    if (x < from.before) from = Search{};
    while (from.at < a.S) {
        const SeqRange r = from.at ? load_range(a, from.at + lane) : first;
        const int64_t n = measure(r);
        int64_t up = n;                        // inclusive scan over the lanes
        for (int m = 1; m < lanes; m <<= 1) {
            const int64_t y = __shfl_up(up, m, WAVE);
            if (lane >= m) up += y;
        }
        const uint64_t hit = __ballot(lane < lanes && from.before + up > x);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            f.r.q0 = __builtin_amdgcn_readlane(r.q0, l);
            f.r.qlen = __builtin_amdgcn_readlane(r.qlen, l);
            f.r.klen = __builtin_amdgcn_readlane(r.klen, l);
            f.s = from.at + l;
            f.base = from.before + lane64(up - n, l);
            return true;
        }
        from.before += lane64(up, lanes - 1);
        from.at += 64;
    }
    return false;
}
// The tile of place `pos` of all work, and the tile's place and cost.  Lane by lane: even lanes one pos and odd ones another (a
// share's begin and end at once: it is a chain of a few hundred instructions).
struct Tile { Found f; int32_t g = 0, tile = 0; int64_t start = 0, w = 0; bool many = false; };
__device__ __forceinline__ void tile_of(const AttnArgs& a, const Plan& plan, const SeqRange& first, int64_t pos, Search& from, Tile& t) {
    int32_t g = (int32_t)((float)pos / (float)plan.head);        // about, then exactly
    g = g < a.G ? g : a.G - 1;
    while (g > 0 && g * plan.head > pos) --g;
    while (g < a.G - 1 && (g + 1) * plan.head <= pos) ++g;
    const int64_t x = pos - g * plan.head;
    auto cost = [&](const SeqRange& r) {
        const Line l = seq_line(r, a.Hg, a.causal, a.window, a.costs);
        return line_before(l, l.tiles);
    };
    Found odd;
    const int64_t x0 = lane64(x, 0), x1 = lane64(x, 1);
    find(a, first, x0, from, t.f, cost);
    odd = t.f;
    if (x1 != x0) {
        Search other;
        find(a, first, x1, other, odd, cost);
    }
    const bool second = threadIdx.x & 1;
    SeqRange r;
    r.q0 = second ? odd.r.q0 : t.f.r.q0;
    r.qlen = second ? odd.r.qlen : t.f.r.qlen;
    r.klen = second ? odd.r.klen : t.f.r.klen;
    const int64_t base = second ? odd.base : t.f.base;
    const Line l = seq_line(r, a.Hg, a.causal, a.window, a.costs);
    t.g = g;
    t.tile = line_tile(l, x - base);
    t.start = g * plan.head + base + line_before(l, t.tile);
    t.w = line_at(l, t.tile);
    t.many = is_many(r, a.Hg);
}
// What the second launch is told of a share: where it begins, in which tile (that one's place), and whether inside it.
struct Share { int64_t pos, start; SeqRange r; int32_t g, tile, inside; };
// behind the partial rows: into how many shares the work is divided, then these
__device__ __forceinline__ int32_t* among_of(const AttnArgs& a) { return (int32_t*)(a.rec + a.rec_rows * (D + 2)); }
__device__ __forceinline__ Share* shares_of(const AttnArgs& a) { return (Share*)(among_of(a) + 4); }
constexpr size_t SHARES_BYTES = 16 + SLOTS * sizeof(Share);

template <typename ET>
struct Form {
    static constexpr bool BF = sizeof(ET) == 2;
    static constexpr int ROWB = D * (int)sizeof(ET);       // bytes of a row
    static constexpr int PPR = ROWB / 16;
    static constexpr int NF = BF ? 8 : 16;                 // 16-byte fragments of a row per lane: pieces 2 k + h
    static constexpr int NC = BF ? 2 : 1;                  // many rows: blocks of 32 rows per wave
    static constexpr int WAVES = ROWS_MANY / (32 * NC);    // 4; fp32 8, two a SIMD
    static constexpr int KB = 32 * ROWB;
    // many rows: 4 stages of 16 KB of keys, then as many of values; every wave brings LPW KB of either
    static constexpr int SB = 16384;
    static constexpr int KT = SB / ROWB;                   // keys per stage: 64, fp32 32
    static constexpr int SPS = KT / 32;                    // 32-key steps per stage
    static constexpr int STAGES = 4;
    static constexpr int LPW = SB / 1024 / WAVES, WROWS = LPW * 1024 / ROWB;
    static constexpr size_t LDS = 128 * 1024;
    static_assert(SB == SPS * KB, "steps follow each other");
    static_assert(STAGES * 2 * SB <= (int)LDS, "of the largest");
};

// What both forms need of a piece, and the operations on 32-key blocks.
template <typename ET>
struct Piece {
    typedef Form<ET> F;
    const AttnArgs& a;
    SeqRange r;
    int32_t g, lo, hi;                                     // KV head; keys of the piece
    const uint8_t *kbase, *vbase;                          // the head's rows of page 0
    const int32_t* trow;
    int64_t head_bytes;
    int lane, l32, h;
    uint32_t off0, kaddr;

    __device__ __forceinline__ Piece(const AttnArgs& a_, const Found& f, int g_, int32_t lo_, int32_t hi_, int lane_)
        : a(a_), r(f.r), g(g_), lo(lo_), hi(hi_), lane(lane_) {
        head_bytes = (int64_t)F::ROWB << a.shift;
        kbase = (const uint8_t*)a.k + (int64_t)g * head_bytes;
        vbase = (const uint8_t*)a.v + (int64_t)g * head_bytes;
        trow = a.table + (int64_t)f.s * a.table_stride;
        l32 = lane & 31;
        h = lane >> 5;
        const int lrow = lane / F::PPR;                    // the row that this lane loads of a 1 KB piece
        off0 = (uint32_t)(lrow * F::ROWB + ((lane % F::PPR) ^ ((lrow & 3) << 2)) * 16);
        kaddr = key_addr(lane);
    }
    static __device__ __forceinline__ uint32_t key_addr(int ln) {
        const int row = ln & 31;
        return (uint32_t)(row * F::ROWB + ((ln >> 5) ^ (((row & 3) << 2) | ((row >> 2) & 3))) * 16);
    }
    // the same piece with the lane's numbers anew: what the rare masked steps derive from them is not kept in
    // registers for the whole loop
    __device__ __forceinline__ Piece anew() const {
        Piece p = *this;
        asm volatile("" : "+v"(p.lane), "+v"(p.l32), "+v"(p.h));
        return p;
    }
    // the page of key t as the table has it (any entry of the sequence's behind its end)
    __device__ __forceinline__ int32_t raw_page(int32_t t) const { return trow[(t < r.klen ? t : r.klen - 1) >> a.shift]; }
    // and -1 for one that names none, and behind the end
    __device__ __forceinline__ int32_t page_of(int32_t raw, int32_t t) const {
        return t < r.klen ? good_page(raw, a.n_pages) : -1;
    }
    // where the rows from t on of page p lie in a head's rows of the pool
    __device__ __forceinline__ int64_t offset_of(int32_t p, int32_t t) const {
        return (int64_t)p * a.G * head_bytes + (int64_t)(t & ((1 << a.shift) - 1)) * F::ROWB;
    }
    // rows from t on of page p (or zeros): address of the first, and the advance per 1 KB
    __device__ __forceinline__ const uint8_t* rows_at(const uint8_t* pool, int32_t p, int32_t t) const {
        return (const uint8_t*)first_lane((int64_t)(p >= 0 ? pool + offset_of(p, t) : (const uint8_t*)pa_zeros));
    }
    static __device__ __forceinline__ int advance(int32_t p) { return p >= 0 ? 1024 : 0; }
    // 1 KB number v of them into LDS at dst (of number 0); row 0 of number 0 is row 4 `quad` of its block
    template <bool VALUES, bool ONCE = false>
    __device__ __forceinline__ void bring1(const uint8_t* src, int adv, int v, int quad, uint32_t dst) const {
        // rows 4 v + .. (bf16) or 2 v + .. (fp32): the rest of f(row); fp32 values are read a row at a time as they are
        if constexpr (F::BF) lds_load<ONCE>(src + v * adv, off0 ^ (((uint32_t)(quad + v) & 3u) << 4), dst + v * 1024);
        else if constexpr (!VALUES)
            lds_load<ONCE>(src + v * adv, off0 ^ ((uint32_t)((v & 1) << 3 | ((quad + (v >> 1)) & 3)) << 4), dst + v * 1024);
        else lds_load<ONCE>(src + v * adv, 16u * (uint32_t)lane, dst + v * 1024);
    }
    // values behind the end in the rows [r0, r1) of a tile of keys from t0 on: not read as data
    __device__ __forceinline__ void clear_tail(int32_t t0, int32_t r0, int32_t r1, uint8_t* vt) const {
        const int32_t end = r.klen - t0, stop = (end + 15) & ~15;
        const int32_t from = end > r0 ? end : r0, to = stop < r1 ? stop : r1;
        for (int i = lane; i < (to - from) * F::PPR; i += 64)
            *reinterpret_cast<uint4*>(vt + (from + i / F::PPR) * F::ROWB + (i % F::PPR) * 16) = uint4{0, 0, 0, 0};
    }
    // a row's query as B operand
    __device__ __forceinline__ void query(u32x4 (&qf)[F::NF], int64_t token, int head) const {
        const uint8_t* src = (const uint8_t*)((const ET*)a.q + token * a.q_stride + (int64_t)head * D);
#pragma unroll
        for (int k = 0; k < F::NF; ++k) qf[k] = load16(src + (2 * k + h) * 16);
    }
    // scores of NC blocks of 32 rows with 32 keys
    template <int NC>
    __device__ __forceinline__ void scores(const uint8_t* kt, const u32x4 (&qf)[NC][F::NF], f32x16 (&sc)[NC]) const {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[c][i] = 0.f;
        if constexpr (F::BF) {
#pragma unroll
            for (int k = 0; k < F::NF; ++k) {
                const u32x4 f = *reinterpret_cast<const u32x4*>(kt + (kaddr ^ (32u * k)));
#pragma unroll
                for (int c = 0; c < NC; ++c) sc[c] = mfma32(f, qf[c][k], sc[c]);
            }
        } else {
            const uint32_t ka = key_addr(lane_now());
            u32x4 f[2];
            f[0] = *reinterpret_cast<const u32x4*>(kt + ka);
#pragma unroll
            for (int k = 0; k < F::NF; ++k) {              // the next fragment is read before the products of this one
                if (k + 1 < F::NF)
                    f[(k + 1) & 1] = *reinterpret_cast<const u32x4*>(kt + (ka ^ (32u * ((k + 1) & 7))) + 256 * ((k + 1) >> 3));
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        sc[c] = mfma32(__uint_as_float(f[k & 1][e]), __uint_as_float(qf[c][k][e]), sc[c]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    // The keys that a row sees of this piece, as the first and their number; gm: 16-key groups with a page.
    struct Seen { int32_t lo, n; };
    __device__ __forceinline__ Seen seen(int32_t row_lo, int32_t row_hi) const {
        const int32_t b = row_lo > lo ? row_lo : lo, e = row_hi < hi ? row_hi : hi;
        return Seen{b, e > b ? e - b : 0};
    }
    static __device__ __forceinline__ bool sees(int32_t t, Seen s) { return (uint32_t)(t - s.lo) < (uint32_t)s.n; }
    __device__ __forceinline__ void mask(f32x16& sc, int32_t t0, Seen s, uint32_t gm) const {
        if (gm != 3u) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(gm >> (i >> 3) & 1u)) sc[i] = -INFINITY;
        }
        const uint32_t at = (uint32_t)(t0 + 4 * h - s.lo);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (at + 8 * (i >> 2) + (i & 3) >= (uint32_t)s.n) sc[i] = -INFINITY;
    }
    __device__ __forceinline__ float most(const f32x16& sc) const {
        float m = sc[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) m = fmaxf(m, sc[i]);
        return xmax32(m);
    }
    // V^T fragment, bf16: keys r0 + 4 h + 0..3 and r0 + 8 + 4 h + 0..3, dim 32 dt + l32
    __device__ __forceinline__ u32x4 vfrag(const uint8_t* vt, int r0, int dt) const {
        const int i16 = lane & 15, dh = (lane >> 4) & 1;
        u32x4 f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int row = r0 + 8 * e + 4 * h + (i16 >> 2);
            const int place = (4 * dt + 2 * dh + ((i16 >> 1) & 1)) ^ (((i16 >> 2) << 2) | (2 * e + h));
            const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) pa_s16x4*)(vt + row * F::ROWB + place * 16 + (i16 & 1) * 8)));
            f[2 * e] = v.x;
            f[2 * e + 1] = v.y;
        }
        return f;
    }
    // x with infinities and NaN made 0: one fp32, or a bf16 pair
    static __device__ __forceinline__ uint32_t finite(uint32_t x) {
        if constexpr (F::BF) return x & ~((((x & 0x7F807F80u) + 0x00800080u) >> 15 & 0x00010001u) * 0xFFFFu);
        else return (x & 0x7F800000u) == 0x7F800000u ? 0u : x;
    }
    // acc += V^T P^T of 32 keys; p: the weights, packed in pairs for bf16.  FINITE: of their finite values alone.
    template <int NC, bool FINITE = false>
    __device__ __forceinline__ void values(const uint8_t* vt, const u32x4 (&p)[NC][2], f32x16 (&acc)[NC][4]) const {
#pragma unroll
        for (int mm = 0; mm < 2; ++mm)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                u32x4 f = vfrag(vt, 16 * mm, dt);
                if constexpr (FINITE)
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[k] = finite(f[k]);
#pragma unroll
                for (int c = 0; c < NC; ++c) acc[c][dt] = mfma32(f, p[c][mm], acc[c][dt]);
            }
    }
    // fp32: a lane reads dims 4 l32 .. of key 8 (i / 4) + 4 h + i % 4, one for each of acc, and the next key's before
    // its products: acc[e][n] is dim 4 (8 (n / 4) + 4 h + n % 4) + e.  odd: finite values alone.
    __device__ __forceinline__ void values(const uint8_t* vt, const f32x16& p, f32x16 (&acc)[4], bool odd) const {
        const int ln = lane_now();
        const uint8_t* row = vt + 4 * (ln >> 5) * F::ROWB + 16 * (ln & 31);
        u32x4 f[2];
        f[0] = *reinterpret_cast<const u32x4*>(row);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i < 15) f[(i + 1) & 1] = *reinterpret_cast<const u32x4*>(row + (8 * ((i + 1) >> 2) + ((i + 1) & 3)) * F::ROWB);
            __builtin_amdgcn_sched_barrier(0);
            if (odd)
#pragma unroll
                for (int e = 0; e < 4; ++e) f[i & 1][e] = finite(f[i & 1][e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = mfma32(__uint_as_float(f[i & 1][e]), p[i], acc[e]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // A masked block whose values hold infinities or NaN: 0 x inf is not 0, so a row must not meet the values of keys
    // that it does not see.  The products take the finite values, and every row adds the others of the keys that it sees.
    __device__ __forceinline__ bool odd_values(const uint8_t* vt) const {
        uint32_t odd = 0;
        for (int i = lane; i < F::KB / 16; i += 64) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(vt + 16 * i);
#pragma unroll
            for (int k = 0; k < 4; ++k) odd |= w[k] ^ finite(w[k]);
        }
        return __ballot(odd != 0) != 0;
    }
    // add(dt, i, x): x to the lane's sum of dim 32 dt + 8 (i / 4) + 4 h + i % 4, fp32 32 dt + 16 h + i
    template <typename A>
    __device__ __forceinline__ void add_odd(const uint8_t* vt, int32_t t0, Seen s, uint32_t gm, A&& add) const {
#pragma unroll 1
        for (int kk = 0; kk < 32; ++kk) {
            const bool see = sees(t0 + kk, s) && (gm >> (kk >> 4) & 1u);
            const int f = F::BF ? ((kk & 3) << 2) | ((kk >> 2) & 3) : 0;
#pragma unroll
            for (int n = 0; n < 16; ++n) {                 // four dims
                const int byte = (F::BF ? 8 * n + 4 * h : 32 * (n >> 2) + 16 * h + 4 * (n & 3)) * (int)sizeof(ET);
                const uint8_t* at = vt + kk * F::ROWB + (((byte >> 4) ^ f) << 4) + (byte & 15);
                float x[4];
                if constexpr (F::BF) {
                    const uint2 w = *reinterpret_cast<const uint2*>(at);
                    const uint2 o = {w.x ^ finite(w.x), w.y ^ finite(w.y)};   // the others alone
                    x[0] = bf_lo(o.x);
                    x[1] = bf_hi(o.x);
                    x[2] = bf_lo(o.y);
                    x[3] = bf_hi(o.y);
                } else {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(w[k] ^ finite(w[k]));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) add(n >> 2, 4 * (n & 3) + k, see ? x[k] : 0.f);
            }
        }
    }
};

// weights exp2(c x + off) of 32 keys, in place (fp32), or rounded to bf16 and packed in pairs, which is what the value products
// take, and summed as rounded: a row whose weights are all rounded one way is not off by it.  rest: -1 for what the rounding
// takes from the weights, rounded, in their place; 0 for the weights.
__device__ __forceinline__ void weights(f32x16& sc, float c, float off, float rest, u32x4 (&p)[2], float& l) {
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * k], c, off)), e1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * k + 1], c, off));
        uint32_t w = cvt_bf16x2(e0, e1);
        w = cvt_bf16x2(fmaf(rest, bf_lo(w), e0), fmaf(rest, bf_hi(w), e1));
        p[k >> 2][k & 3] = w;
        if (k & 1) l1 = add_pair(w, l1);
        else l0 = add_pair(w, l0);
    }
    l += l0 + l1;
}
__device__ __forceinline__ float weight32(float x, float c, float c_lo, float off) {
    return __builtin_amdgcn_exp2f(fmaf(x, c_lo, fmaf(x, c, off)));
}
// how: a score's weight
template <typename W>
__device__ __forceinline__ void weights32(f32x16& sc, float& l, W&& how) {
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        sc[i] = how(sc[i]);
        sc[i + 1] = how(sc[i + 1]);
        l0 += sc[i];
        l1 += sc[i + 1];
    }
    l += l0 + l1;
}

// A row's running maximum m (of raw scores) and its sum; a key's weight is exp2(c x + off), off = -c m.  The maximum that
// the weights are taken against follows the true one only when that is SLACK powers of two above it: the weights
// then reach 2^SLACK, which neither bf16's exponent nor the fp32 sums mind, and the sums are rescaled
// a few times per piece instead of at every block.
constexpr float SLACK = 8.f;                               // (SLACK / c is less than half a step of a maximum BEYOND)
// off is rounded, as it is used everywhere (no part of a fused operation): weights of different maxima then differ by
// exp2 of the difference of their offs, whose own roundings cancel.  That rounding and c's (c_lo) leave c m + off up to
// 2^-22 |c m| from 0, a factor that all of the row's weights share.  From |c m| = BEYOND on it would no longer be a number
// to multiply with, and scores next to each other lie 2^-24 |c m| >= 16 apart: the largest takes all.  c is then a power
// of two that takes m to 2^31 .. 2^32 (m's own exponent is 0 exactly, the next score's below -127), whether or not c m
// itself is within fp32's range.
constexpr float BEYOND = 0x1.1p28f;
__device__ __forceinline__ bool beyond(float off) { return fabsf(off) >= BEYOND; }
__device__ __forceinline__ float power_for(float m) { return __uint_as_float((uint32_t)(159 - __builtin_amdgcn_frexp_expf(m)) << 23); }
__device__ __forceinline__ float off_of(float m, float c) {
    float off = m == -INFINITY ? 0.f : -m * c;             // 0 while nothing has been seen
    asm("" : "+v"(off));
    return beyond(off) ? -m * power_for(m) : off;          // exact; -infinity for m = infinity, whose weight is NaN
}
// the factor that takes sums of weights against m to those against M >= m, whose off is `to`
__device__ __forceinline__ float factor(float m, float off, float M, float to) {
    const float f = __builtin_amdgcn_exp2f(to - off);
    return m == -INFINITY || (m != M && (beyond(off) || beyond(to))) ? 0.f : f;
}
__device__ __forceinline__ float rescale(float m, float M, float to, float c) { return factor(m, off_of(m, c), M, to); }
struct Running {
    float m = -INFINITY, off = 0.f, l = 0.f;
    // the factor for what has been summed so far
    __device__ __forceinline__ float raise(float mt, float c) {
        const float mn = fmaxf(m, mt), to = off_of(mn, c), f = factor(m, off, mn, to);
        m = mn;
        off = to;
        l *= f;
        return f;
    }
    // the c that a row's weights take (c, c_lo: the call's)
    __device__ __forceinline__ float c_of(float c) const { return beyond(off) ? power_for(m) : c; }
    // a weight of fp32 layers where some row of the wave is beyond (the others keep both parts of c)
    __device__ __forceinline__ float weight_of(float x, float c, float c_lo) const {
        return beyond(off) ? __builtin_amdgcn_exp2f(fmaf(x, power_for(m), off)) : weight32(x, c, c_lo, off);
    }
};

template <typename ET>
__device__ __forceinline__ void store4(ET* dst, float o0, float o1, float o2, float o3) {
    if constexpr (sizeof(ET) == 2) *reinterpret_cast<uint2*>(dst) = uint2{cvt_bf16x2(o0, o1), cvt_bf16x2(o2, o3)};
    else *reinterpret_cast<f32x4*>(dst) = f32x4{o0, o1, o2, o3};
}

// Few rows: rows 0 .. rows - 1 of the sequence's one tile.
template <typename ET>
__device__ void few_rows(const Piece<ET>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row);

// Many rows, what bf16 and fp32 share: rows row0 .. row0 + rows - 1 of the sequence, 32 NC of them a wave,
// the key stages and which steps of 32 keys the wave's rows see.
template <typename ET>
struct Many {
    typedef Form<ET> F;
    static constexpr int NC = F::NC;
    const Piece<ET>& P;
    uint8_t* smem;
    uint32_t lds0;
    int wave, crow;                                        // crow: the first of the wave's rows of a stage
    int32_t row0, rows, wrow, t_first, stages;
    int32_t jf, jl, mf, ml;                                // steps that some row sees: [jf, jl), every row whole: [mf, ml)
    // pages of the 16-key groups of a window of 64 groups, one a lane: the one that is being brought, the raw
    // entries of the next, and which groups of the last two windows have a page
    static constexpr int SPW = 1024 / F::KT;               // stages per window
    int32_t raw;
    const uint8_t *kwin, *vwin;                            // of the window: its groups' first rows
    uint64_t has[2];
    bool bad;                                              // some key before the end has had none
    const uint8_t *ksrc, *vsrc;                            // of the stage that is being brought
    int adv;
    uint32_t dst;

    __device__ __forceinline__ Many(const Piece<ET>& P_, uint8_t* smem_, int32_t row0_, int32_t rows_)
        : P(P_), smem(smem_), row0(row0_), rows(rows_) {
        const AttnArgs& a = P.a;
        lds0 = first_lane((int)(uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)smem);
        wave = first_lane((int)(threadIdx.x >> 6));
        crow = wave * F::WROWS;
        wrow = 32 * NC * wave;
        t_first = P.lo & ~(F::KT - 1);
        stages = P.hi > P.lo ? (P.hi - t_first + F::KT - 1) / F::KT : 0;
        jf = jl = mf = ml = 0;
        raw = 0;
        kwin = vwin = nullptr;
        has[0] = has[1] = 0;
        bad = false;
        ksrc = vsrc = nullptr;
        adv = 0;
        dst = 0;
        const int32_t n = rows - wrow < 32 * NC ? rows - wrow : 32 * NC;
        if (n > 0) {
            int32_t lo0, hi0, lo1, hi1;
            row_keys(P.r, (row0 + wrow) / a.Hg, a.causal, a.window, lo0, hi0);
            row_keys(P.r, (row0 + wrow + n - 1) / a.Hg, a.causal, a.window, lo1, hi1);
            jf = first_lane(within(lo0) >> 5);
            jl = first_lane((within(hi1) + 31) >> 5);
            mf = first_lane((within(lo1) + 31) >> 5);
            ml = first_lane(within(hi0) >> 5);
        }
    }
    // token (of the sequence) and query head of lane l32's row of block c, and the keys that it sees
    __device__ __forceinline__ void row_of(int c, int l32, int32_t& tok, int32_t& head) const {
        const int32_t i = wrow + 32 * c + l32, row = row0 + (i < rows ? i : 0);
        tok = row / P.a.Hg;
        head = P.g * P.a.Hg + row % P.a.Hg;
    }
    __device__ __forceinline__ typename Piece<ET>::Seen keys_seen(int c) const {
        int32_t tok, head, lo, hi;
        row_of(c, P.l32, tok, head);
        row_keys(P.r, tok, P.a.causal, P.a.window, lo, hi);
        return P.seen(lo, hi);
    }
    __device__ __forceinline__ int32_t within(int32_t t) const { return (t < P.lo ? P.lo : t > P.hi ? P.hi : t) - t_first; }
    __device__ __forceinline__ int32_t window_key(int w) const { return t_first + 1024 * w + 16 * P.lane; }
    // stage s is to be brought: its addresses ...
    __device__ __forceinline__ void aim(int s) {
        const int w = s / SPW, in = s % SPW;
        if (in == 0) {                                     // a new window: its entries were asked for half a window ago
            if (w == 0) raw = P.raw_page(window_key(0));
            const int32_t t = window_key(w), page = P.page_of(raw, t);
            const uint64_t m = __ballot(page >= 0);
            bad = bad || __ballot(page < 0 && t < P.r.klen) != 0;
            kwin = page >= 0 ? P.kbase + P.offset_of(page, t) : (const uint8_t*)pa_zeros;
            vwin = page >= 0 ? P.vbase + P.offset_of(page, t) : (const uint8_t*)pa_zeros;
            if (w & 1) has[1] = m;
            else has[0] = m;
        }
        if (in == SPW / 2) raw = P.raw_page(window_key(w + 1));
        const int group = (in * F::KT + crow) / 16;
        adv = (w & 1 ? has[1] : has[0]) >> group & 1 ? 1024 : 0;
        const int rest = adv ? crow % 16 * F::ROWB : 0;
        ksrc = (const uint8_t*)lane64((int64_t)kwin, group) + rest;
        vsrc = (const uint8_t*)lane64((int64_t)vwin, group) + rest;
        dst = lds0 + (s & 3) * F::SB + wave * F::LPW * 1024;
    }
    // ... and its loads, the keys' first
    __device__ __forceinline__ void bring(int i) const {
        if (i < F::LPW) P.template bring1<false>(ksrc, adv, i, crow / 4, dst);
        else P.template bring1<true>(vsrc, adv, i - F::LPW, crow / 4, dst + F::STAGES * F::SB);
    }
    __device__ __forceinline__ void bring_half(bool keys) const {
        const uint8_t* src = keys ? ksrc : vsrc;
        const uint32_t to = keys ? dst : dst + F::STAGES * F::SB;
        static_assert(F::BF || F::LPW == 2, "bf16 alone: both kinds of rows are laid out alike");
#pragma unroll
        for (int i = 0; i < F::LPW; ++i) P.template bring1<false>(src, adv, i, crow / 4, to);
    }
    __device__ __forceinline__ void issue(int s) {
        aim(s);
#pragma unroll
        for (int i = 0; i < 2 * F::LPW; ++i) bring(i);
    }
    __device__ __forceinline__ void begin() {
        issue(0);
        issue(1);
    }
    // Stage s has arrived, and stage s - 2 is free (every wave is past it): stage s + 2 follows.  Every stage is
    // followed by others, so that the counts stay the same; those behind the last bring rows that nothing reads.
    __device__ __forceinline__ void arrive(int s) const {
        wait_loads<2 * F::LPW>();
        P.clear_tail(t_first + s * F::KT, crow, crow + F::WROWS, smem + (F::STAGES + (s & 3)) * F::SB);
        __syncthreads();
    }
    __device__ __forceinline__ void finish() const {
        wait_loads<0>();
        __syncthreads();                                   // the stages are free again
    }
    // which 16-key groups of step j have a page (j within two windows of what is being brought)
    __device__ __forceinline__ uint32_t gm_of(int j) const {
        return (uint32_t)((j >> 5 & 1 ? has[1] : has[0]) >> (2 * (j & 31))) & 3u;
    }
    __device__ __forceinline__ uint8_t* keys_of(int j) const { return smem + ((uint32_t)j * F::KB & (F::STAGES * F::SB - 1)); }
    __device__ __forceinline__ uint8_t* values_of(int j) const { return keys_of(j) + F::STAGES * F::SB; }
    __device__ __forceinline__ bool masked(int j) const { return j < mf || j >= ml || gm_of(j) != 3u; }
    // block c's rows: sums (of 32 dims dt, four at a time as the products leave them) and, with `last`, maximum and sum
    __device__ __forceinline__ void put(int c, int dt, const f32x16& o, const Running& run, float l, bool cut, int64_t rec_row,
                                        bool last) const {
        const AttnArgs& a = P.a;
        const int i0 = wrow + 32 * c + P.l32;
        if (i0 >= rows) return;
        const int first = 32 * dt + (F::BF ? 4 : 16) * P.h;
        constexpr int next = F::BF ? 2 : 1;
        if (cut) {
            float* dst = a.rec + (rec_row + i0) * D + first;
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<f32x4*>(dst + next * i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
            if (last && P.h == 0) *reinterpret_cast<float2*>(a.rec + a.rec_rows * D + (rec_row + i0) * 2) = float2{run.m, l};
        } else {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            int32_t tok, head;
            row_of(c, P.l32, tok, head);
            ET* dst = (ET*)a.out + (int64_t)(P.r.q0 + tok) * a.out_stride + (int64_t)head * D + first;
#pragma unroll
            for (int i = 0; i < 16; i += 4) store4<ET>(dst + next * i, o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv);
        }
    }
};

template <typename ET>
__device__ void many_rows(const Piece<ET>& P, uint8_t* smem, int32_t row0, int32_t rows, bool cut, int64_t rec_row);

// grid: at most one workgroup per slot, a multiple of 8.  Whole tiles: a workgroup takes one of each round, half of
// them go through the rounds backwards, so that the single tokens' reads and the chunks' products overlap (of more than 64
// sequences none, so that they are looked through once).  Shares: the work is laid end to end and divided evenly; shares
// that begin or end inside a tile leave partial rows.
//   Even shares, against pieces of one length per call dealt out in turn: 1003 tokens beside 16 single ones 192 -> 173 us
//   (chunk and single tokens side by side from the start), fp32 prompts of 1531 and 777 tokens 339 -> 257 us, 32 single tokens
//   over 100 .. 21800 311 -> 287 us.  Finding a share's ends takes 3 us, which tiles alike in equal pieces save.
//   Where a wave stands lies in shared memory while it works on a piece: kept in scalar registers it spills into the
//   loops' (512 tokens over 32768: 294 -> 283 us).
struct Walk {
    SeqRange first[64];
    Plan plan;
    Search from;
    Tile t;
    int64_t pos, end;
    int32_t place;
};
template <typename ET>
__global__ __launch_bounds__(64 * Form<ET>::WAVES, 1) void paged_attn_kernel(AttnArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(16) uint8_t walks[Form<ET>::WAVES * sizeof(Walk)];
    const uint32_t b = blockIdx.x, n = gridDim.x;
    Walk& w = reinterpret_cast<Walk*>(walks)[first_lane((int)(threadIdx.x >> 6))];
    {
        const SeqRange first = load_range(a, threadIdx.x & 63);
        const Plan plan = wave_plan(a, first);
        if (a.rec_rows && b == 0 && threadIdx.x == 0) *among_of(a) = plan.split.among;
        const int32_t share = share_of(b, plan.split.among);
        if (plan.split.among && share == plan.split.among) return;
        w.first[threadIdx.x & 63] = first;
        w.plan = plan;
        w.from = Search{};
        w.t = Tile{};
        w.pos = w.end = 0;
        w.place = 2 * share;
    }
    for (int k = 0;; ++k) {
        asm volatile("" ::: "memory");                     // read it again
        const SeqRange first = w.first[threadIdx.x & 63];
        const Plan plan = {first_lane(w.plan.head), first_lane(w.plan.units),
                           Split{first_lane(w.plan.split.among), first_lane(w.plan.split.same)}};
        const Split split = plan.split;
        Search from;
        from.at = first_lane(w.from.at);
        from.before = first_lane(w.from.before);
        Tile t;
        int32_t place = first_lane(w.place);
        const int32_t share = place >> 1;
        int64_t x0 = 0, x1 = 0;
        bool cut = false;
        if (split.among && !split.same) {
            const int64_t total = plan.head * a.G;
            t.f.r = SeqRange{first_lane(w.t.f.r.q0), first_lane(w.t.f.r.qlen), first_lane(w.t.f.r.klen)};
            t.f.s = first_lane(w.t.f.s);
            t.g = first_lane(w.t.g);
            t.tile = first_lane(w.t.tile);
            t.start = first_lane(w.t.start);
            t.w = first_lane(w.t.w);
            int64_t pos = first_lane(w.pos), end = first_lane(w.end);
            if (k > 0 && pos >= end) break;
            if (k == 0 || pos >= t.start + t.w) {
                const int64_t at = k ? pos : share_begin(total, share + (int)(threadIdx.x & 1), split);
                Tile u;
                tile_of(a, plan, first, at < total ? at : total - 1, from, u);
                if (k == 0) {                              // where the share begins and ends
                    const int64_t to = at < total ? u.start + cut_at(at - u.start, u.w, u.many, a.costs) : total;
                    w.pos = pos = lane64(to, 0);
                    w.end = end = lane64(to, 1);
                }
                t.f = u.f;
                t.g = first_lane(u.g);
                t.tile = first_lane(u.tile);
                t.start = first_lane(u.start);
                t.w = first_lane(u.w);
                w.t = t;
                w.from = from;
                if (k == 0) {
                    if (threadIdx.x == 0)
                        shares_of(a)[share] = Share{pos, t.start, t.f.r, t.g, t.tile, pos > t.start && pos < t.start + t.w};
                    continue;
                }
            }
            x0 = pos - t.start;
            x1 = end - t.start < t.w ? end - t.start : t.w;
            cut = x1 - x0 != t.w;
            w.pos = t.start + x1;
            w.place = place | 1;
        } else {
            // tiles by their numbers: whole ones sequence after sequence, the last tile first (with causal rows it sees the
            // most keys), heads innermost; those in equal pieces head after head
            const int64_t all = (plan.units + n - 1) / n;
            const int32_t rounds = split.same ? 1 : all < INT32_MAX ? (int32_t)all : INT32_MAX;
            if (k == rounds) break;
            const int32_t G = split.same ? 1 : a.G;
            int64_t idx = tile_number(b, n, b & 8 && a.S <= 64 ? rounds - 1 - k : k);
            if (split.same) {
                const uint32_t u = (uint32_t)share / (uint32_t)split.same, each = (uint32_t)plan.units / (uint32_t)a.G;
                cut = true;
                t.start = u;
                t.w = split.same;
                x0 = share - (int64_t)u * split.same;
                x1 = x0 + 1;
                t.g = (int32_t)(u / each);
                idx = u % each;
            }
            const bool found = find(a, first, idx, from, t.f, [&](const SeqRange& r) { return (int64_t)seq_tiles(r, a.Hg) * G; });
            w.from = from;
            if (!found) continue;                          // behind the last
            const uint32_t in = (uint32_t)(idx - t.f.base);
            if (!split.same) t.g = (int32_t)(in % (uint32_t)G);
            t.tile = seq_tiles(t.f.r, a.Hg) - 1 - (int32_t)(in / (uint32_t)G);
            if (split.same && threadIdx.x == 0)
                shares_of(a)[share] = Share{share, t.start * t.w, t.f.r, t.g, t.tile, x0 != 0};
        }
        const int64_t rec_row = (int64_t)place * place_rows(a.T, a.Hg);
        const SeqRange r = t.f.r;
        const int bm = tile_rows(r, a.Hg);
        const int32_t row0 = t.tile * bm;
        const int32_t rows = (int32_t)(seq_rows(r, a.Hg) - row0 < bm ? seq_rows(r, a.Hg) - row0 : bm);
        int32_t lo, hi;
        tile_keys(r, row0, rows, a.Hg, a.causal, a.window, lo, hi);
        if (cut) piece_keys(x0, x1, t.w, lo, hi);
        // What follows from the lane's number is formed for each piece: kept for all of them it spills (one token over 32768,
        // bf16: 38.4 -> 37.0 us).  Not so for many rows of bf16: a prompt of 1000 tokens takes 53 us, and 61 with it.
        lo = first_lane(lo);
        hi = first_lane(hi);
        if (bm == ROWS_FEW) few_rows<ET>(Piece<ET>(a, t.f, t.g, lo, hi, lane_now()), smem, rows, cut, rec_row);
        else many_rows<ET>(Piece<ET>(a, t.f, t.g, lo, hi, Form<ET>::BF ? (int)(threadIdx.x & 63) : lane_now()), smem, row0, rows, cut, rec_row);
    }
}

// One row's pieces p0, p0 + step, .. of np, for NR rows at once by a half wave, NP pieces at a time with a running
// maximum, so that nothing waits for all maxima first.  at(n, p): the partial row of row n and piece p.
template <int NR, int NP, typename A>
__device__ __forceinline__ void join_pieces(const AttnArgs& a, A&& at, int p0, int step, int np, float (&M)[NR], float (&l)[NR],
                                            f32x4 (&o)[NR]) {
    const float* rec_ml = a.rec + a.rec_rows * D;
    const int l32 = threadIdx.x & 31;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        M[n] = -INFINITY;
        l[n] = 0.f;
        o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int p = p0; p < np; p += NP * step) {
        float2 ml[NR][NP];
        f32x4 v[NR][NP];
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                ml[n][k] = float2{-INFINITY, 0.f};
                v[n][k] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (p + k * step < np) {
                    const int64_t rr = at(n, p + k * step);
                    ml[n][k] = *reinterpret_cast<const float2*>(rec_ml + rr * 2);
                    v[n][k] = *reinterpret_cast<const f32x4*>(a.rec + rr * D + 4 * l32);
                }
            }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            float mn = M[n];
#pragma unroll
            for (int k = 0; k < NP; ++k) mn = fmaxf(mn, ml[n][k].x);
            const float to = off_of(mn, a.c), f0 = rescale(M[n], mn, to, a.c);
            M[n] = mn;
            l[n] *= f0;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] *= f0;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const float f = rescale(ml[n][k].x, mn, to, a.c);
                l[n] = fmaf(f, ml[n][k].y, l[n]);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = fmaf(f, v[n][k][e], o[n][e]);
            }
        }
    }
}
// Joins the tiles that were cut.  grid (parts, shares - 1): the workgroups of every share but the first, which have work if
// theirs is the first to begin inside its tile.  A half wave has a row, 16 bytes a lane, or two; of few rows a workgroup
// has one, every eighth piece a half wave.  It is a chain of reads that the other dies have just written, about 2 us each: what helps is
// rows in parallel and loads that are all of use (1003 tokens of 32 heads in 2 pieces: 8 loads of one row's pieces a
// wave, 6 of them for nothing: 26 us; this: 11 us).
template <typename ET>
__global__ __launch_bounds__(256) void paged_join_kernel(AttnArgs a) {
    __shared__ __align__(16) float so[8][D];
    __shared__ float sl[8][2];
    const int i = 1 + (int)blockIdx.y, part = (int)blockIdx.x, parts = (int)gridDim.x;
    const int lane = threadIdx.x & 63, half = threadIdx.x >> 5, l32 = threadIdx.x & 31;
    // all that may be asked for, at once
    const Share* shares = shares_of(a);
    const Share here = shares[i], before = shares[i - 1];
    const int j0 = i + 1 + lane < SLOTS ? i + 1 + lane : SLOTS - 1;
    int32_t next_inside = shares[j0].inside;
    int64_t next_start = shares[j0].start;
    const int32_t among = first_lane(*among_of(a));
    if (i >= among || !first_lane(here.inside)) return;
    const int64_t start = first_lane(here.start);
    if (first_lane(before.inside) && first_lane(before.start) == start) return;
    const SeqRange r = {first_lane(here.r.q0), first_lane(here.r.qlen), first_lane(here.r.klen)};
    const int g = first_lane(here.g), bm = tile_rows(r, a.Hg);
    const int32_t row0 = first_lane(here.tile) * bm;
    const int32_t rows = (int32_t)(seq_rows(r, a.Hg) - row0 < bm ? seq_rows(r, a.Hg) - row0 : bm);
    // its pieces: share i - 1's last, and the first of i, i + 1, .. that begin inside the tile
    int np = 2;
    for (int j = i + 1;; j += 64) {
        const uint64_t on = __ballot(j + lane < among && next_inside && next_start == start);
        if (on != ~0ull) {
            np += __builtin_ctzll(~on);
            break;
        }
        np += 64;
        const int jn = j + 64 + lane < SLOTS ? j + 64 + lane : SLOTS - 1;
        next_inside = shares[jn].inside;
        next_start = shares[jn].start;
    }
    const int64_t pr = place_rows(a.T, a.Hg);
    const int64_t rec0 = (2 * (i - 1) + (first_lane(before.pos) == start ? 0 : 1)) * pr;
    auto piece = [&](int p) { return p == 0 ? rec0 : 2 * (i + p - 1) * pr; };
    auto put = [&](int32_t in, float l, const f32x4& o) {
        const int32_t row = row0 + in;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        ET* dst = (ET*)a.out + (int64_t)(r.q0 + row / a.Hg) * a.out_stride + (int64_t)(g * a.Hg + row % a.Hg) * D + 4 * l32;
        store4<ET>(dst, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    };
    // (rows behind the tile's last are read as they are and dropped)
    if (bm == ROWS_FEW) {
        for (int row = part; row < rows; row += parts) {
            float M[1], l[1];
            f32x4 o[1];
            join_pieces<1, 8>(a, [&](int, int p) { return piece(p) + row; }, half, 8, np, M, l, o);
            __syncthreads();
            *reinterpret_cast<f32x4*>(&so[half][4 * l32]) = o[0];
            if (l32 == 0) {
                sl[half][0] = M[0];
                sl[half][1] = l[0];
            }
            __syncthreads();
            if (half) continue;
            float mx = sl[0][0], ls = 0.f;
            f32x4 os = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 1; k < 8; ++k) mx = fmaxf(mx, sl[k][0]);
            const float to = off_of(mx, a.c);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = rescale(sl[k][0], mx, to, a.c);
                const f32x4 v = *reinterpret_cast<const f32x4*>(&so[k][4 * l32]);
                ls = fmaf(f, sl[k][1], ls);
#pragma unroll
                for (int e = 0; e < 4; ++e) os[e] = fmaf(f, v[e], os[e]);
            }
            put(row, ls, os);
        }
    } else if (np <= 4) {
        for (int mine = 16 * part + 2 * half; mine < rows; mine += 16 * parts) {
            float M[2], l[2];
            f32x4 o[2];
            join_pieces<2, 4>(a, [&](int n, int p) { return piece(p) + mine + n; }, 0, 1, np, M, l, o);
            put(mine, l[0], o[0]);
            if (mine + 1 < rows) put(mine + 1, l[1], o[1]);
        }
    } else {
        for (int mine = 8 * part + half; mine < rows; mine += 8 * parts) {
            float M[1], l[1];
            f32x4 o[1];
            join_pieces<1, 8>(a, [&](int, int p) { return piece(p) + mine; }, 0, 1, np, M, l, o);
            put(mine, l[0], o[0]);
        }
    }
}

// the second launch follows unless the tables are too short for a cut
template <typename ET>
hipError_t launch_paged(const AttnArgs& a, int groups, hipStream_t st) {
    const void* fn = (const void*)paged_attn_kernel<ET>;
    hipError_t e = ensure_lds_limit(fn, Form<ET>::LDS);
    if (e != hipSuccess) return e;
    paged_attn_kernel<ET><<<groups, 64 * Form<ET>::WAVES, Form<ET>::LDS, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess || !a.rec_rows) return e;
    // about 2048 workgroups that have work: many for each of few tiles, of many tiles a few
    const int64_t units = max_units(a.T, a.S, a.G, a.Hg), each = 2048 / (units ? units : 1);
    const unsigned parts = place_rows(a.T, a.Hg) == ROWS_FEW ? (unsigned)(a.T * a.Hg) : each < 8 ? 8 : each < 32 ? (unsigned)each : 32;
    paged_join_kernel<ET><<<dim3(parts, (unsigned)groups - 1), 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_bf16(const AttnArgs& a, int groups, hipStream_t st);
hipError_t launch_paged_f32(const AttnArgs& a, int groups, hipStream_t st);

}  // namespace vr
