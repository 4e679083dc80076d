// Attention of new tokens over pages of e4m3 codes, gfx950: bf16 queries, and the host side of both.  Half of the raw cache's bytes
// bound few rows (one token over 131072 of 8 KV heads: 61 .. 65 us, raw 100), the same products many.
#include "paged8_attn.h"

namespace vr {

template <>
__device__ __forceinline__ void few_rows<Coded<uint16_t>>(const Piece<Coded<uint16_t>>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    few_rows8<uint16_t>(P, smem, rows, cut, rec_row);
}
// bf16, many rows.  As the raw cache's: one wave has a SIMD to itself, matrix and vector work alternate within it, and the
// iteration of step j (32 keys) forms the scores of j, takes the exponentials of j - 1 and adds the values of j - 2.  What is new
// are the conversions: four instructions a fragment, between two pairs of products each, for the fragment after the next pair, so
// that two fragments at a time are decoded and the others are codes still.  2048 tokens over 32768 of 8 KV heads of 4: 975 .. 1050 us by
// the card, 1015 .. 1092 TFLOP/s, as the raw cache's (step by step with the compiler's own order: 3796 us).
//   23 registers of the kernel are spilt, around the loops over a piece's keys: they are read once a piece, two in masked
//   steps too.
//   Measured and not kept: addresses in shared memory formed at each read by one instruction instead of fetched from AGPRs
//   (seven instructions a step fewer: 1010 -> 1035 us).
template <>
__device__ __forceinline__ void many_rows<Coded<uint16_t>>(const Piece<Coded<uint16_t>>& P, uint8_t* smem, int32_t row0, int32_t rows,
                                                           bool cut, int64_t rec_row) {
    typedef Coded<uint16_t> C;
    typedef Form<C> F;
    const AttnArgs& a = P.a;
    Many<C> M(P, smem, row0, rows);
    if (M.stages) M.begin();
    Running run[2];
    float cw[2] = {a.c, a.c};                              // c of the rows' weights
    settle();
    static_for<128>([&](auto i) { agpr_set<i>(0u); });
    {
        u32x4 qf[2][1][8];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            int32_t tok, head;
            M.row_of(c, P.l32, tok, head);
            P.query(qf[c], nullptr, P.r.q0 + tok, head);
        }
        static_for<64>([&](auto i) { agpr_set<QBASE + i>(qf[i / 32][0][i / 4 % 8][i % 4]); });
    }
    settle();
    const Piece<C>::Seen seen[2] = {M.keys_seen(0), M.keys_seen(1)};
    const float slack = SLACK / a.c;
    f32x16 sc[2][2];
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[0][0][i] = sc[0][1][i] = sc[1][0][i] = sc[1][1][i] = -INFINITY;
    u32x4 p[2][2][2];
    float pend[2] = {1.f, 1.f};
    float mx[2] = {-INFINITY, -INFINITY};                  // this lane's maxima of the last step's scores
    float lb[2] = {0.f, 0.f};                              // every second weight's part of the sums
    bool pending = false;
    // Before the weights of step j - 1, after its scores and the value products of j - 3.
    auto follow = [&]() {
        const bool above = __any(mx[0] > run[0].m + slack || mx[1] > run[1].m + slack);
        if (!(above || pending)) return;
        if (pending) {                                     // the products of j - 3 were of the old maximum
            settle();
            static_for<128>([&](auto i) { agpr_set<i>(__float_as_uint(agpr_get<i>() * pend[i / 64])); });
            settle();
            pending = false;
        }
        if (above) {
            pend[0] = run[0].raise(xmax32(mx[0]), a.c);    // and those of j - 2 will be: scaled after them
            pend[1] = run[1].raise(xmax32(mx[1]), a.c);
            cw[0] = run[0].c_of(a.c);
            cw[1] = run[1].c_of(a.c);
            lb[0] *= pend[0];
            lb[1] *= pend[1];
            pending = true;
        }
    };
    auto kcodes = [&](int j, int n) { return *reinterpret_cast<const u32x4*>(M.keys_of(j) + (P.kaddr ^ (32u * n))); };
    auto decode_key = [&](const u32x4 (&w)[4], int k, float s) {
        return k & 1 ? decode8(uint2{w[k >> 1][2], w[k >> 1][3]}, s) : decode8(uint2{w[k >> 1][0], w[k >> 1][1]}, s);
    };
    // two weights of block c of step j - 1 (e: the parity of j): the exponentials, and packing and summing them
    float ea, eb;
    auto weigh = [&](auto par, int c, int k) {
        constexpr int e = decltype(par)::value;
        ea = __builtin_amdgcn_exp2f(fmaf(sc[1 - e][c][2 * k], cw[c], run[c].off));
        eb = __builtin_amdgcn_exp2f(fmaf(sc[1 - e][c][2 * k + 1], cw[c], run[c].off));
    };
    auto pack = [&](auto par, int c, int k) {
        constexpr int e = decltype(par)::value;
        uint32_t w = cvt_bf16x2(ea, eb);                   // what the value products take
        run[c].l += ea;
        lb[c] += eb;
        asm volatile("" : "+v"(w), "+v"(run[c].l), "+v"(lb[c]));     // here, not where they are used
        p[1 - e][c][k >> 2][k & 3] = w;
    };
    // An odd step waits for the stage of the step after it and brings the keys of two stages on, the next even one the values.
    auto stage_ready = [&](int j) {
        const int s = (j + 1) >> 1;
        M.arrive(s);
        M.aim(s + 2);
    };
    // Step j with nothing to mask in j and j - 2.  kw: its key codes, replaced by those of j + 1; kf: the first of them decoded,
    // likewise.  A fragment is decoded before the weights are packed: products are not covered by the compiler's waits.
    auto fast = [&](auto par, int j, u32x4 (&kw)[4], u32x4 (&kf)[2]) {
        constexpr int e = decltype(par)::value;
        f32x16 &s0 = sc[e][0], &s1 = sc[e][1];
        const uint8_t* vt = M.values_of(j - 2);
        const float ks = M.key_scale(j), vs = M.value_scale(j - 2);
        uint2 vw[8];
        u32x4 vf[2];
        static_for<8>([&](auto k) {
            score<k, 0>(s0, kf[k & 1]);
            if constexpr (k == 0) follow();
            weigh(par, 0, k);
            __builtin_amdgcn_sched_barrier(0);
            score<k, 1>(s1, kf[k & 1]);
            vw[k] = P.vcodes(vt, 16 * (k >> 2), k & 3);
            if constexpr (k < 7) kf[(k + 1) & 1] = decode_key(kw, k + 1, ks);
            else vf[0] = decode8(vw[0], vs);
            __builtin_amdgcn_sched_barrier(0);
            pack(par, 0, k);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (e == 1) stage_ready(j);
        const float next = M.key_scale(j + 1);
        mx[0] = mx[1] = -INFINITY;
        static_for<8>([&](auto n) {
            value<n & 3, 0>(vf[n & 1], p[e][0][n >> 2]);
            weigh(par, 1, n);
            if constexpr (n == 2 || n == 4) M.bring(2 * (1 - e) + (n - 2) / 2);
            __builtin_amdgcn_sched_barrier(0);
            value<n & 3, 1>(vf[n & 1], p[e][1][n >> 2]);
            if constexpr (n < 4) kw[n] = kcodes(j + 1, n);
            if constexpr (n < 7) vf[(n + 1) & 1] = decode8(vw[n + 1], vs);
            else kf[0] = decode_key(kw, 0, next);
            __builtin_amdgcn_sched_barrier(0);
            pack(par, 1, n);
            // the scores' last products were issued before the two pairs of value products that have gone
            // by, each product 8 passes long: they are there
            if constexpr (n == 1) asm volatile("" : "+v"(s0), "+v"(s1));
            if constexpr (n >= 2)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i * 6 / 8 == n - 2) {
                        asm volatile("v_max3_f32 %0, %0, %1, %2" : "+v"(mx[0]) : "v"(s0[2 * i]), "v"(s0[2 * i + 1]));
                        asm volatile("v_max3_f32 %0, %0, %1, %2" : "+v"(mx[1]) : "v"(s1[2 * i]), "v"(s1[2 * i + 1]));
                    }
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // any step, as an even one: sc[1] and p[0] are the steps before, and what it forms is moved there
    auto slow = [&](int j) {
        f32x16 &s0 = sc[0][0], &s1 = sc[0][1];
        const std::integral_constant<int, 0> par{};
        const uint8_t* vt = M.values_of(j - 2);
        const bool qk = j >= M.jf && j < M.jl, ex = j - 1 >= M.jf && j - 1 < M.jl, pv = j - 2 >= M.jf && j - 2 < M.jl;
        const Piece<C> L = P.anew();
        u32x4 kf[8], vf[8];
        if (qk) {
            const float ks = M.key_scale(j);
            u32x4 kw[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) kw[n] = kcodes(j, n);
#pragma unroll
            for (int k = 0; k < 8; ++k) kf[k] = decode_key(kw, k, ks);
        }
        bool odd = false;
        if (pv) {
            const float vs = M.value_scale(j - 2);
            odd = M.masked(j - 2) && L.odd_values(vt);
#pragma unroll
            for (int n = 0; n < 8; ++n) vf[n] = decode8(L.vcodes(vt, 16 * (n >> 2), n & 3), vs);
            if (odd)
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) vf[n][k] = L.finite(vf[n][k]);
        }
        follow();
        auto weights_of = [&](int k) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                weigh(par, c, k);
                pack(par, c, k);
            }
        };
        if (qk) {
            asm volatile("s_nop 1" : "+v"(kf[0]), "+v"(kf[1]), "+v"(kf[2]), "+v"(kf[3]), "+v"(kf[4]), "+v"(kf[5]), "+v"(kf[6]), "+v"(kf[7]));
            static_for<8>([&](auto k) {
                score<k, 0>(s0, kf[k]);
                score<k, 1>(s1, kf[k]);
                weights_of(k);                             // of nothing for the first step: scores of -infinity
            });
            asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s0), "+v"(s1));
        } else if (ex) {
#pragma unroll
            for (int k = 0; k < 8; ++k) weights_of(k);
        }
        if (pv) {
            asm volatile("s_nop 1" : "+v"(vf[0]), "+v"(vf[1]), "+v"(vf[2]), "+v"(vf[3]), "+v"(vf[4]), "+v"(vf[5]), "+v"(vf[6]), "+v"(vf[7]));
            static_for<8>([&](auto n) {
                value<n & 3, 0>(vf[n], p[0][0][n >> 2]);
                value<n & 3, 1>(vf[n], p[0][1][n >> 2]);
            });
            if (odd) {
                settle();
                static_for<2>([&](auto c) {
                    f32x16 o[4];
                    static_for<64>([&](auto i) { o[i / 16][i % 16] = 0.f; });
                    L.add_odd(vt, M.t_first + 32 * (j - 2), seen[c], M.gm_of(j - 2),
                              [&](int dt, int i, float x) { o[dt][i] += x; });
                    static_for<64>([&](auto i) { agpr_set<64 * c + i>(__float_as_uint(agpr_get<64 * c + i>() + o[i / 16][i % 16])); });
                });
                settle();
            }
        }
        mx[0] = mx[1] = -INFINITY;
        if (qk) {
            if (M.masked(j))
#pragma unroll
                for (int c = 0; c < 2; ++c) L.mask(sc[0][c], M.t_first + 32 * j, seen[c], M.gm_of(j));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                mx[0] = fmaxf(mx[0], s0[i]);
                mx[1] = fmaxf(mx[1], s1[i]);
            }
        }
        if (j & 1) stage_ready(j);
        if (j > 0) M.bring_half(j & 1);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            sc[1][c] = sc[0][c];
            p[0][c][0] = p[1][c][0];
            p[0][c][1] = p[1][c][1];
        }
        // the copies are written well before the next step's products read them
        asm volatile("s_nop 1" : "+v"(p[0][0][0]), "+v"(p[0][0][1]), "+v"(p[0][1][0]), "+v"(p[0][1][1]));
    };
    const std::integral_constant<int, 0> even{};
    const std::integral_constant<int, 1> odd{};
    if (M.stages) {
        M.arrive(0);
        M.issue(2);
    }
    const int32_t end = M.stages ? 2 * M.stages + 2 : 0;   // one stage's steps more: the last weights and values
    for (int j = 0; j < end;) {
        if (!(j & 1) && j >= M.mf + 2 && j + 1 < M.ml && !M.bad) {
            u32x4 kw[4], kf[2];
#pragma unroll
            for (int n = 0; n < 4; ++n) kw[n] = kcodes(j, n);
            kf[0] = kf[1] = decode_key(kw, 0, M.key_scale(j));
            asm volatile("s_nop 1" : "+v"(kf[0]), "+v"(kf[1]));
            do {
                fast(even, j, kw, kf);
                fast(odd, j + 1, kw, kf);
                j += 2;
            } while (j + 1 < M.ml && !M.bad);
        } else {
            slow(j);
            ++j;
        }
    }
    settle();
    static_for<2>([&](auto c) {
        const float l = xsum32(run[c].l + lb[c]);
        static_for<4>([&](auto dt) {
            f32x16 o;
            static_for<16>([&](auto i) { o[i.value] = agpr_get<16 * (4 * c + dt) + i>(); });
            M.put(c, dt, o, run[c], l, cut, rec_row, dt == 3);
        });
    });
    M.finish();
}

hipError_t launch_paged8_bf16(const AttnArgs& a, int groups, hipStream_t st) { return launch_paged<Coded<uint16_t>>(a, groups, st); }

// ---- host ------------------------------------------------------------------------------------
size_t paged8_attn_ws_bytes(int64_t T, int S, int G, int H, int dtype, int64_t cap) {
    const int64_t rows = max_records8(T, S, G, H / G, cap, costs8_of(dtype == VARRATE_BF16).lmin);
    return rows ? (size_t)rows * (D + 2) * 4 + SHARES_BYTES : 0;
}

hipError_t launch_paged8_attn(const varrate_pages8& pg, const varrate_batch& b, int dtype, const void* q, int64_t q_stride, int H,
                              int causal, int window, float scale, void* out, int64_t out_stride, float* lse, void* ws, hipStream_t st) {
    AttnArgs a = {};
    a.q = q;
    a.out = out;
    a.k = pg.k;
    a.v = pg.v;
    a.kscale = (const uint8_t*)pg.k_scale;
    a.vscale = (const uint8_t*)pg.v_scale;
    a.lse = lse;
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
    a.costs = costs8_of(dtype == VARRATE_BF16);
    split_scale(scale, a.c, a.c_lo);
    a.most_units = max_units(b.T, b.S, pg.G, a.Hg);
    a.rec_rows = max_records8(b.T, b.S, pg.G, a.Hg, a.cap, a.costs.lmin);
    const int groups = max_groups(b.T, b.S, pg.G, a.Hg, a.cap, a.costs.lmin);
    return dtype == VARRATE_BF16 ? launch_paged8_bf16(a, groups, st) : launch_paged8_f32(a, groups, st);
}

}  // namespace vr
