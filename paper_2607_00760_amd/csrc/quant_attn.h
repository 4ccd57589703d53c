// quant_attn.h -- attention over the 8-bit KV cache, every block or a
// selection (mosaic_quant_decode_attention, mosaic_quant_select_attention);
// one source per code format (quant_attn_*.hip).
//
// out = sum_t p_t v_t / sum_t p_t, p_t = exp(scale q.k_t - max), with k_t and
// v_t their codes times their block's scale.  One pass with running maximum
// and sum: a wave takes a block at a time, straight from memory into matrix
// operands.  A code of either format is a value of both 16-bit types: the
// logits' product is of the query's type and exact, the outputs' is of bf16,
// with each weight's 24 bits in three parts (its upper half, what that leaves,
// and what is left then) in rows [part][head] of the left operand, groups of 5
// to 8 heads with the third in a product of its own.  bf16 reaches as far down
// as the exponential does: a block counts as exactly where its weights lie on
// tokens whose codes are zeros.  A block's value scale goes into its weights;
// the unit of a head's sums is a power of two that follows the largest product
// of weight and scale, however far apart the scales are.
//
// The products' layouts ask for 8 tokens of one channel in a lane: values lie
// by channel in the cache, and the rows of the first product are dealt so that
// a lane's logits are consecutive tokens (token (B / 4) (row / 4) + 4 tile +
// row % 4), so no value passes through LDS.
//
// HBM is the bound: 256 bytes of a token, with the next block's loads out
// while one is worked on.
#pragma once
#include <type_traits>

#include "quant_join.h"

namespace mosaic {

namespace {

// Runs of a launch: with up to 256 pairs they and the pairs' rounding fill the
// 512 workgroups that the chip holds once; more pairs take several rounds anyway.
__host__ __device__ __forceinline__ int qa_runs(int pairs) { return pairs <= 256 ? 512 - pairs : 1024; }
// Units of a run at least: two steps a wave, and up to four rather than a
// second workgroup on a compute unit (a step costs 0.8 us, joining a pair's
// runs 2).  us of calls with runs of at least 4 / 8 / 12 / 16 units, 8 kv heads:
//   1 x 1500 tokens          8.2 /  8.7 /  9.2 /  9.9
//   1 x 4117                 9.9 /  9.6 /  9.5 /  9.6
//   8 x 1500                12.1 / 10.8 / 10.8 / 11.3
//   a tenth of 4 x 32785    22.3 / 20.6 / 20.6 / 20.7
constexpr int QA_LEAST = 2 * QA_NWV, QA_FEW = 256;
// A pair of up to 16 units is one run: 380 tokens 8.4 -> 7.4 us when that came.
// Pairs of up to 256 have no more runs than are joined with one round of loads
// (groups of up to 4 heads): 1 x 4117 tokens 9.7 -> 9.3 when that came.
constexpr int QA_ALONE = 16, QA_JOIN = 16;

// 8 codes as fp16
template <int FMT> __device__ __forceinline__ dhf8 codes_f16(uint32_t a, uint32_t b) {
    typedef __attribute__((ext_vector_type(2))) _Float16 h2;
    h2 o[4];
    const uint32_t w[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (FMT == QF_E4M3) {
            o[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
            o[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true);
        } else {                                           // 1024 + (code + 128) has the code's bits, then - 1152
            const uint32_t u = w[i] ^ 0x80808080u;
            const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
            o[2 * i] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
            o[2 * i + 1] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
        }
    }
    dhf8 r;
    __builtin_memcpy(&r, o, 16);
    return r;
}

// 8 codes as bf16: of the format's conversion, or the upper halves of fp32 integers
template <int FMT> __device__ __forceinline__ DMma<1>::v8 codes_bf16(uint32_t a, uint32_t b) {
    uint32_t o[4];
    const uint32_t w[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (FMT == QF_E4M3) {
            o[2 * i] = e4m3x2<1, false>(w[i]);
            o[2 * i + 1] = e4m3x2<1, true>(w[i]);
        } else {
            const uint32_t x0 = __float_as_uint((float)(int8_t)w[i]), x1 = __float_as_uint((float)(int8_t)(w[i] >> 8));
            const uint32_t x2 = __float_as_uint((float)(int8_t)(w[i] >> 16)), x3 = __float_as_uint((float)(int8_t)(w[i] >> 24));
            o[2 * i] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
            o[2 * i + 1] = __builtin_amdgcn_perm(x3, x2, 0x07060302u);
        }
    }
    DMma<1>::v8 r;
    __builtin_memcpy(&r, o, 16);
    return r;
}
template <int FMT, int DT> __device__ __forceinline__ typename DMma<DT>::v8 codes_of(uint32_t a, uint32_t b) {
    if constexpr (DT) return codes_bf16<FMT>(a, b);
    else return codes_f16<FMT>(a, b);
}

template <int FMT, int B> struct QStage {                  // a block in flight
    uint4 k[B / 16][2];                                    // 16 channels of a token each
    uint32_t v[8][B / 16];                                 // B / 4 tokens of a channel each
    float ks, vs;
};

// GP: heads that a part's rows hold, 4 or 8
template <int FMT, int B, int DT, bool SEL, int GP>
__global__ void __launch_bounds__(64 * QA_NWV) __attribute__((amdgpu_waves_per_eu(2)))
k_quant_attn(QCache q, QSel sel, const uint16_t *query, float scale, uint32_t *arrivals, float *part, float *outp) {
    using DM = DMma<DT>;
    constexpr int NT = B / 16, TPQ = B / 4;                // tiles of 16 tokens, tokens of a lane
    constexpr uint32_t PS = 14;                            // weights are below 2 * 2^PS units
    __shared__ __align__(16) float mrg[QA_NWV][16][D + 2];
    __shared__ int last;
    auto blocks = [&](int L) { return SEL ? q_want(L / B, sel.num, sel.den) : L / B; };
    auto units = [&](int L) { return blocks(L) + (L % B != 0); };        // the unfinished block is a pair's last unit
    const QPlan pl = q_plan(q, QShare{qa_runs(q.S * q.H), QA_FEW, QA_LEAST, 2 * QA_LEAST, QA_NWV, 1, QA_ALONE, QA_JOIN}, units, blockIdx.x);
    if (!pl.live) return;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int p = pl.s * q.H + pl.h;
    const int b0 = pl.i * pl.c, b1 = min(blocks(pl.L), b0 + pl.c), rest = min(units(pl.L), b0 + pl.c) > b1 ? pl.L % B : 0;
    const int l16 = tid & 15, q4 = (tid & 63) >> 4;
    const int head = min(l16 & (GP - 1), q.G - 1);         // (columns past the group repeat its last head)
    const uint16_t *qp = query + ((uint64_t)p * q.G + head) * D;
    const int32_t *list = SEL ? sel.list + (uint64_t)p * q.N : nullptr;
    const uint64_t pb = (uint64_t)p * q.N;
    auto load = [&](int id, QStage<FMT, B> &st) {
        const uint64_t blk = pb + (uint32_t)id;
        const uint8_t *kp = q.k + blk * (B * D), *vp = q.v + blk * (B * D);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                st.k[n][j] = *(const uint4 *)(kp + (TPQ * (l16 >> 2) + 4 * n + (l16 & 3)) * D + 64 * j + 16 * q4);
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) __builtin_memcpy(st.v[ct], __builtin_assume_aligned(vp + (16 * ct + l16) * B + TPQ * q4, TPQ), TPQ);
        st.ks = q.ks[blk];
        st.vs = q.vs[blk];
    };
    QStage<FMT, B> st0, st1;
    int t = b0 + wave;
    // the wave's blocks of this step and the next (a selection's are read one
    // step ahead of their loads; past the run's end the last again)
    auto block_at = [&](int u) { return SEL ? list[min(u, b1 - 1)] : min(u, b1 - 1); };
    int id0 = 0, id1 = 0;
    if (t < b1) { id0 = block_at(t); id1 = block_at(t + QA_NWV); }
    // q operand: column l16 is head l16 % GP, inner index (j, half, q4, i) channel 64 j + 16 q4 + 8 half + i
    typename DM::v8 qb[4];
    float zs = scale * 1.44269504088896340736f;            // softmax scale in powers of two, and q's
    {
        uint16_t w[4][8];
#pragma unroll
        for (int e = 0; e < 4; ++e) __builtin_memcpy(w[e], __builtin_assume_aligned(qp + 64 * (e >> 1) + 16 * q4 + 8 * (e & 1), 16), 16);
        __builtin_amdgcn_sched_barrier(0);
        if (t < b1) load(id0, st0);                        // on its way while q is looked at
        __builtin_amdgcn_sched_barrier(0);
        if (DT) {                                          // largest magnitude in [1, 2): products with codes stay in range
            float x[4][8], a = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 8; ++i) { x[e][i] = h2f(w[e][i], DT); a = fmaxf(a, fabsf(x[e][i])); }
            a = rows_all(a, [](float m, float o) { return fmaxf(m, o); });
            const uint32_t e = min(max(__float_as_uint(a) >> 23, 1u), 253u);
            const float down = __uint_as_float((254u - e) << 23);
            zs *= __uint_as_float(e << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 8; ++i) qb[e][i] = (typename DM::el)(x[e][i] * down);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) __builtin_memcpy(&qb[e], w[e], 16);
        }
    }
    float m_run = -INFINITY, l_run = 0.0f;                 // head l16 % GP; the sum over this lane's tokens only
    float top = 0x1p-100f;                                 // the largest product of weight and value scale so far, of head
                                                           // l16 % GP; acc is in units of the power of two below it, / 2^PS
    auto expo = [](float x) { return max(__float_as_uint(x) >> 23, PS + 1u); };
    auto unit = [&](float x) { return __uint_as_float((expo(x) - PS) << 23); };                // of acc
    auto per_unit = [&](float x) { return __uint_as_float((254u + PS - expo(x)) << 23); };     // its reciprocal
    df4 acc[8];                                            // [channel tile][row 4 q4 + r]
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) acc[ct] = df4{0.0f, 0.0f, 0.0f, 0.0f};
    // the softmax's step over logits z, to products of weight and value scale;
    // returns what takes them to acc's units.  (What follows in 16 bits reaches
    // further than its scale of 1, and has room for a smaller unit: low, least.)
    auto weigh = [&](float (&z)[NT][4], float vs, float reach, float low, float least) {
        float cm = -INFINITY;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) cm = fmaxf(cm, z[n][r]);
        cm = rows_all(cm, [](float a, float b) { return fmaxf(a, b); });
        const float mn = fmaxf(m_run, cm);
        const float mb = mn == -INFINITY ? 0.0f : mn;
        const float alpha = __builtin_amdgcn_exp2f(m_run - mb);
        float ls = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float e = __builtin_amdgcn_exp2f(z[n][r] - mb);
                ls += e;
                z[n][r] = e * vs;
            }
        l_run = fmaf(l_run, alpha, ls);
        m_run = mn;
        const float was = unit(top);
        top = fmaxf(fmaxf(top * alpha, __builtin_amdgcn_exp2f(cm - mb) * reach) * low, least);
        const float per = per_unit(top), grow = alpha * was * per;
        if (!__all(grow == 1.0f)) {                        // some head's running maximum or unit moved
            float f[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {                  // grow of head (4 q4 + r) % GP
                const float a0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(grow), r));
                const float a1 = GP == 4 ? a0 : __int_as_float(__builtin_amdgcn_readlane(__float_as_int(grow), 4 + r));
                f[r] = (q4 & 1) ? a1 : a0;
            }
#pragma unroll
            for (int ct = 0; ct < 8; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[ct][r] *= f[r];
        }
        return per;
    };
    // the left operand of tokens 8 s + [0, 8) of the lane's; with GP = 8 the third
    // parts are an operand of their own, in the first parts' rows
    auto split = [&](const float (&z)[NT][4], int s, float per, int l16, dbf8 &pa, dbf8 &third) {
        const uint32_t half1 = l16 >= GP ? 0xffff0000u : 0u, half2 = l16 >= 2 * GP ? 0xffff0000u : 0u, first = l16 < GP ? ~0u : 0u;
        float x[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = z[2 * s + (i >> 2)][i & 3] * per;
            if (GP == 8) {
                const float r = beyond(w);
                x[i] = l16 < GP ? w : r;
                y[i] = __uint_as_float(__float_as_uint(beyond(r)) & first);
            } else {
                x[i] = beyond(beyond(w, half1), half2);
            }
        }
        pa = upper_halves(x);
        if (GP == 8) third = upper_halves(y);
    };
    auto consume = [&](const QStage<FMT, B> &st) {
        float z[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            df4 a = df4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                a = DM::run(codes_of<FMT, DT>(st.k[n][j].x, st.k[n][j].y), qb[2 * j], a);
                a = DM::run(codes_of<FMT, DT>(st.k[n][j].z, st.k[n][j].w), qb[2 * j + 1], a);
            }
            const float f = zs * st.ks;
#pragma unroll
            for (int r = 0; r < 4; ++r) z[n][r] = a[r] * f;          // token TPQ q4 + 4 n + r, head l16 % GP
        }
        const float per = weigh(z, st.vs, st.vs, 1.0f, 0.0f);
#pragma unroll
        for (int s = 0; s < B / 32; ++s) {
            dbf8 pa, third;
            split(z, s, per, l16, pa, third);
#pragma unroll
            for (int ct = 0; ct < 8; ++ct) {
                const dbf8 vb = codes_bf16<FMT>(st.v[ct][2 * s], st.v[ct][2 * s + 1]);
                acc[ct] = DMma<1>::run(pa, vb, acc[ct]);
                if (GP == 8) acc[ct] = DMma<1>::run(third, vb, acc[ct]);
            }
        }
    };
    while (t < b1) {                                       // (two steps a turn: no copies that would wait on the loads)
        load(id1, st1);
        id0 = block_at(t + 2 * QA_NWV);
        __builtin_amdgcn_sched_barrier(0);
        consume(st0);
        t += QA_NWV;
        if (t >= b1) break;
        load(id0, st0);
        id1 = block_at(t + 2 * QA_NWV);
        __builtin_amdgcn_sched_barrier(0);
        consume(st1);
        t += QA_NWV;
    }
    if (rest && wave == ((b1 - b0) & (QA_NWV - 1))) {      // the unfinished block, in 16 bits
        using M8 = typename DM::v8;
        int at = tid;                                      // (worked out again: nothing of it lives through the loop)
        asm volatile("" : "+v"(at));
        const int l16 = at & 15, q4 = (at & 63) >> 4;
        const uint16_t *qp = query + ((uint64_t)p * q.G + min(l16 & (GP - 1), q.G - 1)) * D;
        const uint16_t *kp = q.kt + (uint64_t)p * B * D, *vp = q.vt + (uint64_t)p * B * D;
        M8 qd[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) __builtin_memcpy(&qd[e], qp + 32 * e + 8 * q4, 16);
        uint4 vt[B / 32][8];                               // (rows behind the last token may hold anything)
#pragma unroll
        for (int s = 0; s < B / 32; ++s)
#pragma unroll
            for (int ct = 0; ct < 8; ++ct) {
                const int keep = rest - (TPQ * q4 + 8 * s);    // tokens of the lane's eight
                uint4 x = *(const uint4 *)(vp + (16 * ct + l16) * B + TPQ * q4 + 8 * s);
                x.x = keep >= 2 ? x.x : (keep == 1 ? x.x & 0xffffu : 0u);
                x.y = keep >= 4 ? x.y : (keep == 3 ? x.y & 0xffffu : 0u);
                x.z = keep >= 6 ? x.z : (keep == 5 ? x.z & 0xffffu : 0u);
                x.w = keep >= 8 ? x.w : (keep == 7 ? x.w & 0xffffu : 0u);
                vt[s][ct] = x;
            }
        float z[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            df4 a = df4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                M8 x;
                __builtin_memcpy(&x, kp + (TPQ * (l16 >> 2) + 4 * n + (l16 & 3)) * D + 32 * e + 8 * q4, 16);
                a = DM::run(x, qd[e], a);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                z[n][r] = TPQ * q4 + 4 * n + r < rest ? a[r] * (scale * 1.44269504088896340736f) : -INFINITY;
        }
        // fp16 values are at most 2^16 of a unit and leave their sums room.  bf16
        // ones go up to 2^128: the unit knows the largest, and is 2^60 below it, as
        // the weights' parts would fall below 2^-126 next to the largest values.
        float reach = 1.0f;
        if (DT) {
            float a = 0.0f;
#pragma unroll
            for (int s = 0; s < B / 32; ++s)
#pragma unroll
                for (int ct = 0; ct < 8; ++ct)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {          // (the lower half adds less than a step to the upper one)
                        const uint32_t w = ((const uint32_t *)&vt[s][ct])[e];
                        a = fmaxf(a, fmaxf(fabsf(__uint_as_float(w)), fabsf(__uint_as_float(w << 16))));
                    }
            reach = __uint_as_float(wave_max_u(__float_as_uint(a)));
        }
        const float per = DT ? weigh(z, 1.0f, reach, 0x1p-60f, 0x1p-60f) : weigh(z, 1.0f, 1.0f, 1.0f, 0.0f);
#pragma unroll
        for (int s = 0; s < B / 32; ++s) {
            dbf8 pa, third;
            split(z, s, per, l16, pa, third);
            auto add = [&](df4 &a, const dbf8 &vb) {
                a = DMma<1>::run(pa, vb, a);
                if (GP == 8) a = DMma<1>::run(third, vb, a);
            };
#pragma unroll
            for (int ct = 0; ct < 8; ++ct) {
                if (DT) {
                    add(acc[ct], __builtin_bit_cast(dbf8, vt[s][ct]));
                } else {                                   // an fp16 value's 11 bits in two parts
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t w = ((const uint32_t *)&vt[s][ct])[i >> 1];
                        x[i] = h2f((uint16_t)((i & 1) ? w >> 16 : w), 0);
                    }
                    add(acc[ct], upper_halves(x));
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = beyond(x[i]);
                    add(acc[ct], upper_halves(x));
                }
            }
        }
    }
    // join the waves
    l_run = rows_all(l_run, [](float a, float b) { return a + b; });
    int lane = tid;
    asm volatile("" : "+v"(lane));
    lane &= 63;
    const int row = lane >> 4, col = lane & 15;   // (worked out again, as above)
    if (lane < 16) {                                       // a head's unit stands in the row of its second parts
        mrg[wave][col][0] = lane < GP ? m_run : unit(top);
        mrg[wave][col][1] = l_run;
    }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) mrg[wave][4 * row + r][2 + 16 * ct + col] = acc[ct][r];
    join_waves<GP, GP == 4 ? 3 : 2, false>(mrg, last, pl, q.G, p, arrivals, part, outp);
}

}  // namespace

template <int FMT>
hipError_t launch_quant_attn_t(const QCache &q, int block, int dtype, const uint16_t *query, float scale, const QSel &sel,
                               void *ws, float *out, hipStream_t s) {
    const int pairs = q.S * q.H, runs = qa_runs(pairs) + pairs;
    uint32_t *arrivals = (uint32_t *)ws;
    float *part = (float *)(arrivals + 2 * Q_RUNS);
    const int units = (sel.list ? q_want(q.N, sel.num, sel.den) : q.N) + 1;
    const long long most = (long long)pairs * ceil_div(units, QA_LEAST);
    const dim3 grid((uint32_t)(most < runs ? most : runs));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * QA_NWV), 0, s, q, sel, query, scale, arrivals, part, out); };
    auto by_group = [&](auto b, auto dt, auto selected) {
        constexpr int BL = decltype(b)::value, T = decltype(dt)::value;
        constexpr bool SL = decltype(selected)::value;
        if (q.G <= 4) go(k_quant_attn<FMT, BL, T, SL, 4>); else go(k_quant_attn<FMT, BL, T, SL, 8>);
    };
    auto by_list = [&](auto b, auto dt) { if (sel.list) by_group(b, dt, std::true_type{}); else by_group(b, dt, std::false_type{}); };
    auto by_type = [&](auto b) { if (dtype) by_list(b, std::integral_constant<int, 1>{}); else by_list(b, std::integral_constant<int, 0>{}); };
    if (block == 32) by_type(std::integral_constant<int, 32>{}); else by_type(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

}  // namespace mosaic
