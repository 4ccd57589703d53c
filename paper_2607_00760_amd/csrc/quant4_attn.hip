// quant4_attn.hip -- decode attention over the 4-bit KV cache
// (mosaic_nibble_decode_attention).
//
// out = sum_t p_t v_t / sum_t p_t, p_t = exp(scale q.k_t - max), with
// k_tc = zk_c + sk_c a_tc and v_tc = zv_t + sv_t b_tc, codes a and b of 0 to 15:
//   q.k_t = sum_c q_c zk_c + sum_c (q_c sk_c) a_tc
//   sum_t p_t v_tc = sum_t p_t (zv_t + 8 sv_t) + sum_t (p_t sv_t) (b_tc - 8)
// so no value is worked out: scales go into the query's copy of the block and
// into the weights, once for all tokens and for all channels.  (The middle of a
// token's values is taken apart, not their least: sums over many tokens stay as
// small as their result, and so do their roundings.)  One pass with running
// maximum and sum; a wave takes a block at a time, straight from memory into
// matrix operands; only the grids pass through LDS, as 16 lanes share them.
//
// The logits' product is bf16: a code of 0 to 15 is, as an E4M3 byte, the number
// itself times 2^-9, which one instruction turns into bf16 for two codes.  q_c
// sk_c has 16 bits in bf16 and 22 in fp16: two or three bf16 parts in columns
// [part][head] of the right operand.  The outputs' product is fp16: a code's
// bits under 1024 are 1024 + code, which an addition centres; a weight is two
// fp16 parts in rows [part][head] of the left operand.  So both products are
// exact up to the sums' fp32 roundings and 2^-23 of a weight.
//
// What bounds it: 8 x 128 K tokens of 8 heads, groups of 4 (1.17 GB) 253 us, 4.6
// TB/s, a copy's rate being 4.95, with the vector ALU 65 % busy; 16 ragged
// sequences of up to 96 K tokens, 4 heads, groups of 7, blocks of 32 (0.57 GB) 149
// us, 3.8 TB/s: eight rows of weights a code instead of four and grids twice as
// often, so the ALU is the bound.  fp16, groups of 5 to 8, has the third parts of the
// query in a product of their own: the ragged case 168 us, 8 x 128 K with groups of 8
// 279.  One sequence of 4117 tokens 10.5 us, a chain of
// plan, query, two steps and joins.
//
// The second sum is in units of a power of two that follows the largest product
// of a weight and a token's scale, so weights keep to fp16's range however far
// apart scales are (a unit of the largest weight times the largest scale lost
// weights of 2^-30 on values 2^40 times as large as the others'); the first is in
// units of its own, so bf16 values may be of any size.
#include <type_traits>

#include "quant4.h"
#include "quant_join.h"

namespace mosaic {

namespace {

// Runs of a launch, as in the 8-bit cache's attention: they fill the 512 workgroups
// that the chip holds once.
__host__ __device__ __forceinline__ int q4_runs(int pairs) { return pairs <= 256 ? 512 - pairs : 1024; }
// Units of a run at least: a step a wave, and up to four rather than a second
// workgroup on a compute unit.  us of calls, 8 kv heads, blocks of 64, with runs of
// 4 to 16 units / 8 to 16 / 12 to 24 / 4 to 8:
//   1 x 1500 tokens      9.0 / 11.1 / 12.8 /  9.0
//   1 x 4117            10.7 / 10.8 / 12.3 / 10.8
//   4 x 8192            15.6 / 15.6 / 15.7 / 18.2
// A pair of up to 512 tokens is one run: 380 (blocks of 32) 8.1, and 9.1 with two;
// 1000 (blocks of 64) 12.2 as one, 11.1 with two, 8.8 with four.
constexpr int Q4_LEAST = QA_NWV, Q4_MUCH = 4 * QA_NWV, Q4_FEW = 256, Q4_JOIN = 16;
template <int B> constexpr int Q4_ALONE = 512 / B;

template <int B> struct Q4Stage {                          // a block in flight
    uint4 k[B / 16];                                       // 32 channels of a token each
    uint32_t v[8][B / 32];                                 // B / 4 tokens of a channel each
    uint4 g;                                               // lanes 0..31: the keys' grids, then the values'
};

// the codes of w as bf16, in the order 0, 2, 4, 6, 1, 3, 5, 7
__device__ __forceinline__ dbf8 k_codes(uint32_t w) {
    const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
    uint32_t o[4];
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
    dbf8 r;
    __builtin_memcpy(&r, o, 16);
    return r;
}
__device__ __forceinline__ constexpr int k_order(int i) { return (2 * i & 7) + (i >> 2); }

// the codes of w less 8 as fp16, in the order 0, 4, 1, 5, 2, 6, 3, 7
// (`base`: 0x64006400 from a vector register, as one instruction takes its mask
// and its other constant from nowhere else.)
__device__ __forceinline__ dhf8 v_codes(uint32_t w, uint32_t base) {
    typedef __attribute__((ext_vector_type(2))) _Float16 h2;
    const h2 off = {(_Float16)1032.0f, (_Float16)1032.0f}, by = {(_Float16)0.0625f, (_Float16)0.0625f}, off16 = {(_Float16)-72.0f, (_Float16)-72.0f};
    h2 o[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t u = e ? w >> 8 : w;
        o[2 * e] = __builtin_bit_cast(h2, (u & 0x000f000fu) | base) - off;
        o[2 * e + 1] = __builtin_elementwise_fma(__builtin_bit_cast(h2, (u & 0x00f000f0u) | base), by, off16);
    }
    dhf8 r;
    __builtin_memcpy(&r, o, 16);
    return r;
}
__device__ __forceinline__ constexpr int v_order(int i) { return (i >> 1) + 4 * (i & 1); }

__device__ __forceinline__ const uint32_t *words(const uint4 *x) { return (const uint32_t *)x; }

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
__device__ __forceinline__ uint32_t pk_umax(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int ROR> __device__ __forceinline__ float ror_add(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + ROR, 0xf, 0xf, false));
}

// GP: heads that a part's rows and columns hold, 4 or 8
template <int B, int DT, int GP>
__global__ void __launch_bounds__(64 * QA_NWV) __attribute__((amdgpu_waves_per_eu(2)))
k_quant4_attn(Q4Cache q, const uint16_t *query, float scale, uint32_t *arrivals, float *part, float *outp) {
    using DM = DMma<DT>;
    using M8 = typename DM::v8;
    constexpr int NT = B / 16, TPQ = B / 4, NS = B / 32;   // tiles of 16 tokens, tokens of a lane, steps of the second product
    constexpr uint32_t PS = 14;                            // weights are below 2 * 2^PS units
    constexpr bool THIRD = GP == 8 && !DT;                 // third parts of the query are an operand of their own
    __shared__ __align__(16) float mrg[QA_NWV][16][D + 2];
    __shared__ uint4 grids[QA_NWV][(2 * D + 2 * B) / 8];   // a wave's block: scales and zeros of channels, of tokens
    __shared__ int last;
    auto units = [&](int L) { return (L + B - 1) / B; };   // the unfinished block is a pair's last unit
    const QPlan pl = q_plan(q, QShare{q4_runs(q.S * q.H), Q4_FEW, Q4_LEAST, Q4_MUCH, QA_NWV, 1, Q4_ALONE<B>, Q4_JOIN}, units, blockIdx.x);
    if (!pl.live) return;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int p = pl.s * q.H + pl.h;
    const int whole = pl.L / B, b0 = pl.i * pl.c, b1 = min(whole, b0 + pl.c), rest = min(units(pl.L), b0 + pl.c) > b1 ? pl.L % B : 0;
    const int l16 = tid & 15, q4 = (tid & 63) >> 4;
    const int head = min(l16 & (GP - 1), q.G - 1);         // (columns past the group repeat its last head)
    const uint16_t *qp = query + ((uint64_t)p * q.G + head) * D;
    const uint64_t pb = (uint64_t)p * q.N;
    auto load = [&](int id, Q4Stage<B> &st) {
        const uint64_t blk = pb + (uint32_t)id;
        const uint8_t *kp = q.k + blk * (B * D / 2), *vp = q.v + blk * (B * D / 2);
        constexpr int KG = 2 * D / 8, VG = 2 * B / 8;      // lanes that take the keys' grids, and the values'
        const int lane = tid & 63;
        const uint16_t *g = lane < KG ? q.kg + blk * (2 * D) + 8 * lane : q.vg + blk * (2 * B) + 8 * min(lane - KG, VG - 1);
        st.g = *(const uint4 *)g;
#pragma unroll
        for (int n = 0; n < NT; ++n) st.k[n] = *(const uint4 *)(kp + (TPQ * (l16 >> 2) + 4 * n + (l16 & 3)) * (D / 2) + 16 * q4);
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) __builtin_memcpy(st.v[ct], __builtin_assume_aligned(vp + (16 * ct + l16) * (B / 2) + TPQ / 2 * q4, TPQ / 2), TPQ / 2);
    };
    Q4Stage<B> st0, st1;
    int t = b0 + wave;
    // the query's channels 32 q4 + 8 e + [0, 8), head l16 % GP
    uint4 qw[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) qw[e] = *(const uint4 *)(qp + 32 * q4 + 8 * e);
    if (t < b1) load(t, st0);
    const float zs = powers_of(scale);
    const uint32_t flip = flip_of(scale), keep = scale == 0.0f ? 0u : ~0u;
    auto scaled = [&](uint4 w) { return make_uint4((w.x & keep) ^ flip, (w.y & keep) ^ flip, (w.z & keep) ^ flip, (w.w & keep) ^ flip); };
#pragma unroll
    for (int e = 0; e < 4; ++e) qw[e] = scaled(qw[e]);
    // the part of the query's products that the lane's column holds
    const int mypart = GP == 8 ? l16 >> 3 : (DT ? (l16 >> 2) & 1 : l16 >> 2);
    const uint32_t qh1 = mypart >= 1 ? 0xffff0000u : 0u, qh2 = mypart >= 2 ? 0xffff0000u : 0u, qh3 = mypart >= 3 ? 0u : ~0u;
    float m_run = -INFINITY, l_run = 0.0f;                 // head l16 % GP; sums over this lane's tokens only
    float shift = 0.0f;                                    // sum of p (zv + 8 sv), for bf16 in units of far's power of two
    float top = 0x1p-100f, far = 0x1p-100f;                // the largest product of a weight and a scale so far, and a bound of
                                                           // one and a zero; units are the powers of two below them, / 2^PS
    auto expo = [](float x) { return max(__float_as_uint(x) >> 23, PS + 1u); };
    auto unit = [&](float x) { return __uint_as_float((expo(x) - PS) << 23); };
    auto per_unit = [&](float x) { return __uint_as_float((254u + PS - expo(x)) << 23); };
    uint32_t base = 0x64006400u;
    asm volatile("" : "+v"(base));
    df4 acc[8];                                            // [channel tile][row 4 q4 + r]
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) acc[ct] = df4{0.0f, 0.0f, 0.0f, 0.0f};
    // the softmax's step over logits z, to weights: returns what older sums are
    // multiplied by, and the largest weight
    auto weigh = [&](float (&z)[NT][4], float &most) {
        float cm = -INFINITY;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) cm = fmaxf(cm, z[n][r]);
        cm = rows_all(cm, [](float a, float b) { return fmaxf(a, b); });
        const float mn = fmaxf(m_run, cm);
        const float mb = mn == -INFINITY ? 0.0f : mn;
        const float mz = -mb * zs, alpha = __builtin_amdgcn_exp2f((m_run - mb) * zs);
        most = __builtin_amdgcn_exp2f((cm - mb) * zs);
        float ls = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                z[n][r] = __builtin_amdgcn_exp2f(fmaf(z[n][r], zs, mz));
                ls += z[n][r];
            }
        l_run = fmaf(l_run, alpha, ls);
        m_run = mn;
        return alpha;
    };
    // the unit of the sums follows to `reach`; returns what takes products to it.
    // (What follows in 16 bits has room for a smaller unit: low, least.)
    auto follow = [&](float alpha, float reach, float low, float least) {
        const float was = unit(top);
        top = fmaxf(fmaxf(top * alpha, reach) * low, least);
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
    // the left operand of eight weights in units, in two fp16 parts (11 bits, and
    // the next 11)
    const uint32_t wh = (l16 & GP) ? 0xffffe000u : 0u;
    auto split16 = [&](const float (&w)[8]) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(beyond(w[2 * i], wh), beyond(w[2 * i + 1], wh)));
        dhf8 r;
        __builtin_memcpy(&r, o, 16);
        return r;
    };
    auto consume = [&](const Q4Stage<B> &st) {
        uint4 *lg = grids[wave];
        mem_fence_compiler();
        if ((tid & 63) < (2 * D + 2 * B) / 8) lg[tid & 63] = st.g;
        mem_fence_compiler();
        wave_sync();
        dbf8 qa[4], qt[4];                                 // the query's products with the block's scales
        df4 zq = df4{0.0f, 0.0f, 0.0f, 0.0f};              // what the zeros add
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint4 ks = lg[4 * q4 + e], kz = lg[D / 8 + 4 * q4 + e];
            M8 zo, qo;
            __builtin_memcpy(&zo, &kz, 16);
            __builtin_memcpy(&qo, &qw[e], 16);
            zq = DM::run(zo, qo, zq);
            float x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = half_of<DT>(words(&qw[e]), k_order(i)) * half_of<DT>(words(&ks), k_order(i));
                if (THIRD) {
                    const float r = beyond(w);
                    x[i] = mypart ? r : w;
                    y[i] = __uint_as_float(__float_as_uint(beyond(r)) & (mypart ? 0u : ~0u));
                } else if (DT) {
                    x[i] = beyond(w, qh1);
                } else {
                    x[i] = __uint_as_float(__float_as_uint(beyond(beyond(w, qh1), qh2)) & qh3);
                }
            }
            qa[e] = upper_halves(x);
            if (THIRD) qt[e] = upper_halves(y);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) zq[r] = mypart == 0 ? zq[r] : 0.0f;
        float z[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            df4 a = zq;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const dbf8 c = k_codes(words(&st.k[n])[e]);
                a = DMma<1>::run(c, qa[e], a);
                if (THIRD) a = DMma<1>::run(c, qt[e], a);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {                  // token TPQ q4 + 4 n + r, head l16 % GP: the parts joined
                float s = a[r];
                if (GP == 8 || !DT) s = ror_add<8>(s);
                if (GP == 4) s = ror_add<4>(s);
                z[n][r] = s;
            }
        }
        uint4 vs[NS], vz[NS];                              // of the lane's tokens
#pragma unroll
        for (int s = 0; s < NS; ++s) { vs[s] = lg[2 * D / 8 + NS * q4 + s]; vz[s] = lg[(2 * D + B) / 8 + NS * q4 + s]; }
        float most;
        const float alpha = weigh(z, most);
        float w[NS][8], mids = 0.0f, reach = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = v_order(i);
                const float e = z[2 * s + (at >> 2)][at & 3], sc = half_of<DT>(words(&vs[s]), at);
                w[s][i] = e * sc;
                reach = fmaxf(reach, w[s][i]);
                if (!DT) mids = fmaf(e, fmaf(sc, 8.0f, half_of<DT>(words(&vz[s]), at)), mids);
            }
        if (DT) {                                          // (the sums of a block, too, could pass fp32's range)
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < TPQ / 2; ++i) m = pk_umax(m, pk_umax(words(vs)[i], words(vz)[i] & 0x7fff7fffu));
            const float big = rows_all(fmaxf(half_of<DT>(&m, 0), half_of<DT>(&m, 1)), [](float a, float b) { return fmaxf(a, b); });
            const float was = unit(far);
            far = fmaxf(far * alpha, most * big);
            const float per = per_unit(far);
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    mids = fmaf(z[2 * s + (i >> 2)][i & 3] * per, fmaf(half_of<DT>(words(&vs[s]), i), 8.0f, half_of<DT>(words(&vz[s]), i)), mids);
            shift = fmaf(shift, alpha * was * per, mids);
        } else {
            shift = fmaf(shift, alpha, mids);
        }
        const float per = follow(alpha, rows_all(reach, [](float a, float b) { return fmaxf(a, b); }), 1.0f, 0.0f);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[s][i] *= per;
            const dhf8 pa = split16(w[s]);
#pragma unroll
            for (int ct = 0; ct < 8; ++ct) acc[ct] = DMma<0>::run(pa, v_codes(st.v[ct][s], base), acc[ct]);
        }
    };
    while (t < b1) {                                       // (two steps a turn: no copies that would wait on the loads)
        load(min(t + QA_NWV, b1 - 1), st1);
        __builtin_amdgcn_sched_barrier(0);
        consume(st0);
        t += QA_NWV;
        if (t >= b1) break;
        load(min(t + QA_NWV, b1 - 1), st0);
        __builtin_amdgcn_sched_barrier(0);
        consume(st1);
        t += QA_NWV;
    }
    if (rest && wave == ((b1 - b0) & (QA_NWV - 1))) {      // the unfinished block, in 16 bits
        int at = tid;                                      // (worked out again: nothing of it lives through the loop)
        asm volatile("" : "+v"(at));
        const int l16 = at & 15, q4 = (at & 63) >> 4;
        const uint16_t *qp = query + ((uint64_t)p * q.G + min(l16 & (GP - 1), q.G - 1)) * D;
        const uint16_t *kp = q.kt + (uint64_t)p * B * D, *vp = q.vt + (uint64_t)p * B * D;
        M8 qd[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint4 f = scaled(*(const uint4 *)(qp + 32 * e + 8 * q4));
            __builtin_memcpy(&qd[e], &f, 16);
        }
        uint4 vt[NS][8];                                   // (rows behind the last token may hold anything)
#pragma unroll
        for (int s = 0; s < NS; ++s)
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
            for (int r = 0; r < 4; ++r) z[n][r] = TPQ * q4 + 4 * n + r < rest ? a[r] : -INFINITY;
        }
        // A bf16 product, with three parts of the weights (the third in one of its
        // own) and two of fp16 values.  fp16 values are at most 2^16 of a unit and
        // leave their sums room.  bf16 ones go up to 2^128: the unit knows the largest,
        // and is 2^60 below it, as the parts would fall below 2^-126 next to the
        // largest values.
        float reach = 1.0f, most;
        if (DT) {
            float a = 0.0f;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int ct = 0; ct < 8; ++ct)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {          // (the lower half adds less than a step to the upper one)
                        const uint32_t w = words(&vt[s][ct])[e];
                        a = fmaxf(a, fmaxf(fabsf(__uint_as_float(w)), fabsf(__uint_as_float(w << 16))));
                    }
            reach = __uint_as_float(wave_max_u(__float_as_uint(a)));
        }
        const float alpha = weigh(z, most);
        const float per = DT ? follow(alpha, most * reach, 0x1p-60f, 0x1p-60f) : follow(alpha, most, 1.0f, 0.0f);
        if (DT) {                                          // (shift's unit follows, too)
            const float was = unit(far);
            far *= alpha;
            shift *= alpha * was * per_unit(far);
        } else {
            shift *= alpha;
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float x[8], y[8];
            const uint32_t second = (l16 & GP) ? 0xffff0000u : 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = z[2 * s + (i >> 2)][i & 3] * per;
                x[i] = beyond(w, second);
                y[i] = second ? 0.0f : beyond(beyond(w));
            }
            const dbf8 pa = upper_halves(x), third = upper_halves(y);
            auto add = [&](df4 &a, const dbf8 &vb) {
                a = DMma<1>::run(pa, vb, a);
                a = DMma<1>::run(third, vb, a);
            };
#pragma unroll
            for (int ct = 0; ct < 8; ++ct) {
                if (DT) {
                    add(acc[ct], __builtin_bit_cast(dbf8, vt[s][ct]));
                } else {
                    float u[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = half_of<0>(words(&vt[s][ct]), i);
                    add(acc[ct], upper_halves(u));
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = beyond(u[i]);
                    add(acc[ct], upper_halves(u));
                }
            }
        }
    }
    // join the waves
    l_run = rows_all(l_run, [](float a, float b) { return a + b; });
    shift = rows_all(shift, [](float a, float b) { return a + b; }) * share_of(l_run) * (DT ? unit(far) : 1.0f);   // an average
    int lane = tid;
    asm volatile("" : "+v"(lane));
    lane &= 63;
    const int row = lane >> 4, col = lane & 15;            // (worked out again, as above)
    if (lane < 16) {                                       // a head's unit and shift stand in the row of its second parts
        mrg[wave][col][0] = lane < GP ? m_run * zs : unit(top);
        mrg[wave][col][1] = lane < GP ? l_run : shift;
    }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) mrg[wave][4 * row + r][2 + 16 * ct + col] = acc[ct][r];
    join_waves<GP, 2, true>(mrg, last, pl, q.G, p, arrivals, part, outp);
}

}  // namespace

size_t quant4_attn_ws_bytes(int pairs) {
    return (size_t)2 * Q_RUNS * sizeof(uint32_t) + (size_t)(q4_runs(pairs) + pairs) * QA_PART * sizeof(float);
}

hipError_t launch_quant4_attn(const Q4Cache &q, int block, int dtype, const uint16_t *query, float scale, void *ws, float *out,
                              hipStream_t s) {
    const int pairs = q.S * q.H, runs = q4_runs(pairs) + pairs;
    uint32_t *arrivals = (uint32_t *)ws;
    float *part = (float *)(arrivals + 2 * Q_RUNS);
    const long long most = (long long)pairs * ceil_div(q.N + 1, Q4_LEAST);
    const dim3 grid((uint32_t)(most < runs ? most : runs));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * QA_NWV), 0, s, q, query, scale, arrivals, part, out); };
    auto by_group = [&](auto b, auto dt) {
        constexpr int BL = decltype(b)::value, T = decltype(dt)::value;
        if (q.G <= 4) go(k_quant4_attn<BL, T, 4>); else go(k_quant4_attn<BL, T, 8>);
    };
    auto by_type = [&](auto b) { if (dtype) by_group(b, std::integral_constant<int, 1>{}); else by_group(b, std::integral_constant<int, 0>{}); };
    if (block == 32) by_type(std::integral_constant<int, 32>{}); else by_type(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

}  // namespace mosaic
