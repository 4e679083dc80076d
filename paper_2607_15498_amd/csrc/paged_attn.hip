// Attention of new tokens over a paged cache, gfx950.
//
// o_r = sum_t p_rt v_t / sum_t p_rt,  p_rt = exp(c (x_rt - max_t x_rt)),  x_rt = <q_r, k_t>, over the
// keys t that row r sees, in one pass with a running maximum and sum.  The rows of one KV head are the
// (new token, query head) pairs that read it.  Everything is computed transposed: S^T = K Q^T leaves
// a lane one row (query) and 16 keys of every 32, so maximum and sum are almost wholly within the
// lane, and S^T is already the B operand of O^T = V^T P^T (the keys' order in a product is free, and
// V^T's fragments are read in the order in which S^T holds them).
//
// Two forms, chosen per sequence by its rows.  Few rows (single tokens): the waves of a workgroup
// share one tile of 32 rows and divide its keys, with rings of their own and no barrier, joined at the
// end; the reads of K and V bound it (one token over 131072 of 8 KV heads: 100 us, 5.4 TB/s).  Many rows
// (prompts and chunks): tiles of 256 rows, 64 a wave (two blocks of 32, so that a fragment read from
// LDS feeds two products), and all waves share the key stages; the matrix cores bound it (2048 tokens
// over 32768: 1055 .. 1100 TFLOP/s).  Few are what one product's 32 columns hold: over 32768, 8 tokens of 4
// rows take 41 us (one token 37), 9 as many rows 69, and so do 16: a tile of 256 costs its products however many
// of its rows there are.  In fp32 67 and 180 us.
// One launch serves both, so a chunk and the single tokens beside it run together.  Where there are too
// few (sequence, head, row tile) units for the card, or they are too unlike, their keys are cut (vr_pages.h)
// and a second launch joins the partial rows.
//
// Keys and values come by direct-to-LDS loads of 1 KB (whole rows).  Row r's 16-byte piece c lies at
// place c ^ f(r), f(r) = 4 (r % 4) + (r / 4) % 4, which spreads the K fragment reads (32 rows, one
// piece) and the transposing V reads (8 rows, 4 pieces) over all banks (no conflict is counted); fp32 values, read a row
// at a time, lie as they come.
#include "paged_agpr.h"

namespace vr {

// Few rows: each of the 4 waves takes every fourth tile of 32 keys, out of its own ring of two (16 KB each), and
// their sums are joined at the end.
// Weights are rounded to bf16 for their products with the values.  Up to 16 rows (single tokens) leave half of a product's 32
// columns: these take the same rows' queries, and of their weights what the rounding takes away, so that 2^-16 is missing
// from a row's sums instead of 2^-8 (outputs of a few alike keys were off by up to 7 times their own rounding), for 40 vector
// instructions a tile: 8 x 1 over 16384 61.5 -> 61.7 us, 1 over 32768 37.3 -> 37.7.  (As products of their own, for all 32 rows:
// 64 and 40 us.)
template <>
__device__ __forceinline__ void few_rows<uint16_t>(const Piece<uint16_t>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    typedef uint16_t ET;
    typedef Form<ET> F;
    const AttnArgs& a = P.a;
    const SeqRange& r = P.r;
    const int wave = first_lane((int)(threadIdx.x >> 6)), lane = P.lane, l32 = P.l32, h = P.h;
    const int Hg = a.Hg, g = P.g, lo = P.lo, hi = P.hi;
    constexpr int CH = F::KB / 4096, CROWS = 4096 / F::ROWB;       // a tile's keys (or values) come in chunks of 4 KB
    uint8_t* ring = smem + wave * 4 * F::KB;
    const uint32_t ring0 = first_lane((int)(uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)ring);
    const bool halves = rows <= 16;
    const int col = halves ? l32 & 15 : l32, myrow = col < rows ? col : 0, tok = myrow / Hg;
    const float rest = col < l32 ? -1.f : 0.f;
    int32_t mylo, myhi, firsthi, lastlo, x;
    row_keys(r, tok, a.causal, a.window, mylo, myhi);
    const auto seen = P.seen(mylo, myhi);
    row_keys(r, 0, a.causal, a.window, x, firsthi);
    row_keys(r, (rows - 1) / Hg, a.causal, a.window, lastlo, x);
    u32x4 qf[1][F::NF];
    P.query(qf[0], r.q0 + tok, g * Hg + myrow % Hg);
    Running run;
    const float slack = SLACK / a.c;
    f32x16 acc[1][4], sc[1];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[0][dt][i] = 0.f;

    // pages of the two 16-key groups of the wave's next 32 tiles, one a lane
    constexpr int L = 4 * CH, step = 4 * 32;               // loads of a tile's keys (or values); keys to the next tile
    int32_t window = 0, page[2];
    int at = 32;
    auto fetch = [&](int32_t t) {
        if (at == 32) {
            const int32_t tl = t + (lane >> 1) * step + (lane & 1) * 16;
            window = P.page_of(P.raw_page(tl), tl);
            at = 0;
        }
        page[0] = __builtin_amdgcn_readlane(window, 2 * at);
        page[1] = __builtin_amdgcn_readlane(window, 2 * at + 1);
        ++at;
    };
    auto bring = [&](auto values, const uint8_t* pool, int32_t t, uint32_t dst) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int32_t pg = page[c * CROWS / 16];
            const uint8_t* src = P.rows_at(pool, pg, t + c * CROWS);
#pragma unroll
            for (int v = 0; v < 4; ++v) P.template bring1<values, true>(src, P.advance(pg), v, c * CROWS / 4, dst + c * 4096);
        }
    };
    auto groups = [&]() { return (page[0] >= 0 ? 1u : 0u) | (page[1] >= 0 ? 2u : 0u); };
    int32_t t0 = (lo & ~31) + 32 * wave;
    uint32_t gm_in = 0;
    if (t0 < hi) {
        fetch(t0);
        bring(std::false_type(), P.kbase, t0, ring0);
        bring(std::true_type(), P.vbase, t0, ring0 + F::KB);
        gm_in = groups();
    }
    for (int st = 0; t0 < hi; t0 += step) {
        const uint32_t gm = gm_in;
        uint8_t* kt = ring + st * 2 * F::KB;
        const int32_t tn = t0 + step;
        const bool more = tn < hi;
        const bool masked = t0 < lastlo || t0 < lo || t0 + 32 > firsthi || t0 + 32 > hi || gm != 3u;
        u32x4 p[1][2];
        auto softmax = [&]() {
            P.template scores<1>(kt, qf, sc);
            if (masked) P.anew().mask(sc[0], t0, seen, gm);
            const float mt = P.most(sc[0]);
            if (__any(mt > run.m + slack)) {
                const float f = run.raise(mt, a.c);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[0][dt][i] *= f;
            }
            if (__any(beyond(run.off))) weights(sc[0], run.c_of(a.c), run.off, rest, p[0], run.l);
            else weights(sc[0], a.c, run.off, rest, p[0], run.l);
        };
        st ^= 1;
        const uint32_t next = ring0 + st * 2 * F::KB;
        wait_lds();                                        // the other tile has been read
        if (more) {
            fetch(tn);
            bring(std::false_type(), P.kbase, tn, next);
            bring(std::true_type(), P.vbase, tn, next + F::KB);
            gm_in = groups();
            wait_loads<3 * L>();
        } else wait_loads<L>();
        softmax();
        if (more) wait_loads<2 * L>();
        else wait_loads<0>();
        uint8_t* vt = kt + F::KB;
        P.clear_tail(t0, 0, 32, vt);
        const bool odd = masked && P.anew().odd_values(vt);
        if (odd) {
            P.anew().template values<1, true>(vt, p, acc);
            P.anew().add_odd(vt, t0, seen, gm, [&](int dt, int i, float x) { acc[0][dt][i] += x; });
        } else P.template values<1>(vt, p, acc);
    }
    run.l = xsum32(run.l);
    __syncthreads();                                       // every wave is done with its ring
    float* js = (float*)smem;                              // [4][32][132] sums
    float* jm = js + 4 * 32 * 132;                         // [4][32][2]
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4*>(js + (wave * 32 + l32) * 132 + 32 * dt + 2 * i + 4 * h) =
                f32x4{acc[0][dt][i], acc[0][dt][i + 1], acc[0][dt][i + 2], acc[0][dt][i + 3]};
    if (h == 0) *reinterpret_cast<float2*>(jm + (wave * 32 + l32) * 2) = float2{run.m, run.l};
    __syncthreads();
    // A thread's four times 4 dims: of a row's 16, or of the 8 of a row and of its rests
    const int row = halves ? 4 * wave + (lane >> 4) : 8 * wave + (lane >> 3), d0 = halves ? 8 * (lane & 15) : 16 * (lane & 7);
    const int second = halves ? 16 * 132 : 8;
    if (row < rows) {
        float mw[4], lw[4], M = -INFINITY, Ls = 0.f, o[16];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 v = *reinterpret_cast<const float2*>(jm + (w * 32 + row) * 2);
            mw[w] = v.x;
            lw[w] = v.y;
            if (halves) lw[w] += jm[(w * 32 + row + 16) * 2 + 1];
            M = fmaxf(M, v.x);
        }
        const float to = off_of(M, a.c);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = rescale(mw[w], M, to, a.c);
            Ls = fmaf(f, lw[w], Ls);
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(js + (w * 32 + row) * 132 + d0 + (i & 4) + (i >> 3) * second);
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i + k] = fmaf(f, v[k], o[i + k]);
            }
        }
        if (halves)                                        // (an infinite value times a rest is no number)
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] += fabsf(o[i]) < INFINITY ? o[i + 8] : 0.f;
        if (cut) {
            float* dst = a.rec + (rec_row + row) * D + d0;
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                if (i < 8 || !halves) *reinterpret_cast<f32x4*>(dst + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
            if (d0 == 0) *reinterpret_cast<float2*>(a.rec + a.rec_rows * D + (rec_row + row) * 2) = float2{M, Ls};
        } else {
            const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
            ET* dst = (ET*)a.out + (int64_t)(r.q0 + row / Hg) * a.out_stride + (int64_t)(g * Hg + row % Hg) * D + d0;
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                if (i < 8 || !halves) store4<ET>(dst + i, o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv);
        }
    }
    __syncthreads();                                       // the rings are free again
}

// bf16.  One wave has a SIMD to itself, so matrix and vector work overlap within it.  The iteration of step j
// (32 keys) has two halves: in the first the scores of j are formed while the exponentials of the first block of
// j - 1 are taken and the value fragments of j - 2 are read, in the second the value products of j - 2 while the
// exponentials of the second block and the maximum of j are taken and the key fragments of j + 1 are read; each
// half is 16 products of 32 cycles, about as much vector work, and half of a stage's 8 loads in the second.  A wave
// issues in order, and a product waits for the one before it: between any two stand about 32 cycles of other work
// (two products back to back, then twice as much: 117 cycles a pair instead of 90).  A step that needs a mask, the
// first two and the last two go through the same one after another.
template <>
__device__ __forceinline__ void many_rows<uint16_t>(const Piece<uint16_t>& P, uint8_t* smem, int32_t row0, int32_t rows,
                                                    bool cut, int64_t rec_row) {
    typedef Form<uint16_t> F;
    const AttnArgs& a = P.a;
    Many<uint16_t> M(P, smem, row0, rows);
    if (M.stages) M.begin();
    Running run[2];
    float cw[2] = {a.c, a.c};                              // c of the rows' weights
    settle();
    static_for<128>([&](auto i) { agpr_set<i>(0u); });
    {
        u32x4 qf[2][8];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            int32_t tok, head;
            M.row_of(c, P.l32, tok, head);
            P.query(qf[c], P.r.q0 + tok, head);
        }
        static_for<64>([&](auto i) { agpr_set<QBASE + i>(qf[i / 32][i / 4 % 8][i % 4]); });
    }
    settle();
    const Piece<uint16_t>::Seen seen[2] = {M.keys_seen(0), M.keys_seen(1)};
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
    auto kfrag = [&](int j, int k) { return *reinterpret_cast<const u32x4*>(M.keys_of(j) + (P.kaddr ^ (32u * k))); };
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
        run[c].l += ea;                                    // as they are: the sum of the rounded pair, by whichever
        lb[c] += eb;                                       // instructions, costs 5% (2048 over 32768 980 -> 1041 us)
        asm volatile("" : "+v"(w), "+v"(run[c].l), "+v"(lb[c]));     // here, not where they are used
        p[1 - e][c][k >> 2][k & 3] = w;
    };
    // An odd step waits for the stage of the step after it and brings the first half of two stages on, the next
    // even one the second half.
    auto stage_ready = [&](int j) {
        const int s = (j + 1) >> 1;
        M.arrive(s);
        M.aim(s + 2);
    };
    // step j with nothing to mask in j and j - 2; kf: its key fragments, replaced by those of j + 1
    auto fast = [&](auto par, int j, u32x4 (&kf)[8]) {
        constexpr int e = decltype(par)::value;
        f32x16 &s0 = sc[e][0], &s1 = sc[e][1];
        const uint8_t* vt = M.values_of(j - 2);
        u32x4 vf[8];
        static_for<8>([&](auto k) {
            score<k, 0>(s0, kf[k]);
            if constexpr (k == 0) follow();
            weigh(par, 0, k);
            __builtin_amdgcn_sched_barrier(0);
            score<k, 1>(s1, kf[k]);
            vf[k] = P.vfrag(vt, 16 * (k >> 2), k & 3);
            pack(par, 0, k);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (e == 1) stage_ready(j);
        mx[0] = mx[1] = -INFINITY;
        static_for<8>([&](auto n) {
            value<n & 3, 0>(vf[n], p[e][0][n >> 2]);
            weigh(par, 1, n);
            if constexpr (n >= 2 && n < 6) M.bring(4 * (1 - e) + n - 2);
            __builtin_amdgcn_sched_barrier(0);
            value<n & 3, 1>(vf[n], p[e][1][n >> 2]);
            kf[n] = kfrag(j + 1, n);
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
    // any step, as an even one: sc[1] and p[0] are the steps before, and what it forms is moved there (one copy of
    // the code: short prompts run little else, and fetching it is most of what it costs)
    auto slow = [&](int j) {
        f32x16 &s0 = sc[0][0], &s1 = sc[0][1];
        const std::integral_constant<int, 0> par{};
        const uint8_t* vt = M.values_of(j - 2);
        const bool qk = j >= M.jf && j < M.jl, ex = j - 1 >= M.jf && j - 1 < M.jl, pv = j - 2 >= M.jf && j - 2 < M.jl;
        const Piece<uint16_t> L = P.anew();
        u32x4 kf[8], vf[8];
        if (qk)
#pragma unroll
            for (int k = 0; k < 8; ++k) kf[k] = kfrag(j, k);
        if (pv)
#pragma unroll
            for (int n = 0; n < 8; ++n) vf[n] = L.vfrag(vt, 16 * (n >> 2), n & 3);
        follow();
        auto weights_of = [&](int k) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                weigh(par, c, k);
                pack(par, c, k);
            }
        };
        if (qk) {
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
            const bool odd = M.masked(j - 2) && L.odd_values(vt);
            if (odd) {
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) vf[n][k] = L.finite(vf[n][k]);
                asm volatile("s_nop 3" : "+v"(vf[0]), "+v"(vf[1]), "+v"(vf[2]), "+v"(vf[3]), "+v"(vf[4]), "+v"(vf[5]), "+v"(vf[6]), "+v"(vf[7]));
            }
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
            u32x4 kf[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) kf[k] = kfrag(j, k);
            do {
                fast(even, j, kf);
                fast(odd, j + 1, kf);
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

hipError_t launch_paged_bf16(const AttnArgs& a, int groups, hipStream_t st) { return launch_paged<uint16_t>(a, groups, st); }

// ---- host ------------------------------------------------------------------------------------
size_t paged_attn_ws_bytes(int64_t T, int S, int G, int H, int dtype, int64_t cap) {
    const int64_t rows = max_records(T, S, G, H / G, cap, costs_of(dtype == VARRATE_BF16).lmin);
    return rows ? (size_t)rows * (D + 2) * 4 + SHARES_BYTES : 0;
}

hipError_t launch_paged_attn(const varrate_pages& pg, const varrate_batch& b, const void* q, int64_t q_stride, int H,
                             int causal, int window, float scale, void* out, int64_t out_stride, void* ws, hipStream_t st) {
    AttnArgs a = {};
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
    a.costs = costs_of(pg.dtype == VARRATE_BF16);
    split_scale(scale, a.c, a.c_lo);
    a.most_units = max_units(b.T, b.S, pg.G, a.Hg);
    a.rec_rows = max_records(b.T, b.S, pg.G, a.Hg, a.cap, a.costs.lmin);
    const int groups = max_groups(b.T, b.S, pg.G, a.Hg, a.cap, a.costs.lmin);
    return pg.dtype == VARRATE_BF16 ? launch_paged_bf16(a, groups, st) : launch_paged_f32(a, groups, st);
}

}  // namespace vr
