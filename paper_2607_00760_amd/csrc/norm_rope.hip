// norm_rope.hip -- norms of queries and keys per head and the rotation to
// their positions, in one pass over the rows (mosaic_qk_norm_rope).
//
// Row x of 128 channels, weights w: n = x / sqrt(mean(x^2) + eps) * w, then
// each pair (a, b) of channels is turned by the angle t = position * inv_freq:
// (a cos t - b sin t, b cos t + a sin t).  Everything is fp32 but the angle,
// whose turns position * inv_freq / 2 pi are taken in fp64 and reduced there
// (a position of 2^20 leaves an fp32 angle only 3 digits); results are rounded
// once.
//
// A workgroup takes one token, 16 lanes a row.  A lane holds four whole pairs
// (two pieces of 8 bytes, or one of 16 when interleaved), so nothing is
// exchanged but the sum of squares, four rotations of the 16 lanes.  A lane's
// pairs are the same in every row: the products of weights with sines and
// cosines are made once, and a pair costs six multiplications.  64 lanes
// compute the token's angles while the rows are on their way.  HBM is the
// bound: every row is read and written once.
#include "norm_rope.h"

namespace mosaic {

namespace {

constexpr int NR_ROWS = 16;                                // rows of a workgroup's round
constexpr int NR_AHEAD = 4;                                // rounds of a workgroup at most

template <int ROR> __device__ __forceinline__ float row_ror_add(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + ROR, 0xf, 0xf, false));
}
// over the 16 lanes of a row: the same sum in each
__device__ __forceinline__ float row_sum(float x) {
    x = row_ror_add<8>(x);
    x = row_ror_add<4>(x);
    x = row_ror_add<2>(x);
    return row_ror_add<1>(x);
}

// pair i of a lane's 8 channels: (i, 4 + i), or (2 i, 2 i + 1) when interleaved
template <int DT, bool INTER> __device__ __forceinline__ float2 pair_of(const uint2 (&r)[2], int i) {
    const uint32_t w[4] = {r[0].x, r[0].y, r[1].x, r[1].y};
    if (INTER) return make_float2(h2f((uint16_t)w[i], DT), h2f((uint16_t)(w[i] >> 16), DT));
    const uint32_t a = w[i >> 1], b = w[2 + (i >> 1)];
    return (i & 1) ? make_float2(h2f((uint16_t)(a >> 16), DT), h2f((uint16_t)(b >> 16), DT)) : make_float2(h2f((uint16_t)a, DT), h2f((uint16_t)b, DT));
}
// two fp32 values rounded to the element type (to nearest even; NaN stays NaN)
template <int DT> __device__ __forceinline__ uint32_t pack(float a, float b) {
    if (DT) {
        typedef __attribute__((ext_vector_type(2))) __bf16 b2;
        b2 r;
        r[0] = (__bf16)a;
        r[1] = (__bf16)b;
        return __builtin_bit_cast(uint32_t, r);
    }
    typedef __attribute__((ext_vector_type(2))) _Float16 h2;
    h2 r;
    r[0] = (_Float16)a;
    r[1] = (_Float16)b;
    return __builtin_bit_cast(uint32_t, r);
}

// grid (tokens, rounds of a token's rows / rounds of a workgroup, at most NR_AHEAD)
template <int DT, bool INTER>
__global__ void __launch_bounds__(256) k_norm_rope(NormRope a, int rounds) {
    __shared__ __align__(16) float cs[2][D / 2];
    const int tid = threadIdx.x, l = tid & 15, half = a.half;
    const int64_t s = blockIdx.x / a.n, j = blockIdx.x % a.n;
    const int nrows = a.hq + (a.v ? 2 : 1) * a.hkv, g = (tid & 63) >> 4;
    const int rw0 = blockIdx.y * rounds * NR_ROWS + 4 * __builtin_amdgcn_readfirstlane(tid >> 6);    // the wave's first row
    // the lane's channels c0..c0 + 3 and c1..c1 + 3: pairs (c0 + i, c1 + i), or
    // (c0 + 2 i, c0 + 2 i + 1); lanes past the pairs hold the other channels
    const bool turned = 8 * l < 2 * half;
    const int c0 = INTER || !turned ? 8 * l : 4 * l, c1 = INTER || !turned ? 8 * l + 4 : half + 4 * l;
    uint2 x[NR_AHEAD][2];
    uint16_t *to[NR_AHEAD];
    auto kind_of = [&](int row) { return row < a.hq ? 0 : (row < a.hq + a.hkv ? 1 : 2); };
#pragma unroll
    for (int it = 0; it < NR_AHEAD; ++it) {
        const int rw = rw0 + it * NR_ROWS, row = rw + g;
        if (it < rounds && row < nrows) {
            const uint16_t *src;
            const int kw = kind_of(rw);
            if (kw == kind_of(rw + 3)) {                   // the wave's rows are heads of one kind: scalar addresses, and a
                const NormRope::Part &p = kw == 0 ? a.q : (kw == 1 ? a.k : a.vp);      // lane's head in steps of two strides
                const int h = rw - (kw == 0 ? 0 : (kw == 1 ? a.hq : a.hq + a.hkv));
                src = p.in + (s * p.in_seq + j * p.in_tok + h * p.in_head) + ((g & 1) ? p.in_head : 0) + ((g & 2) ? 2 * p.in_head : 0);
                to[it] = p.out + (s * p.out_seq + j * p.out_tok + h * p.out_head) + ((g & 1) ? p.out_head : 0) + ((g & 2) ? 2 * p.out_head : 0);
            } else {
                const int kind = kind_of(row), h = row - (kind == 0 ? 0 : (kind == 1 ? a.hq : a.hq + a.hkv));
                const NormRope::Part &p = kind == 0 ? a.q : (kind == 1 ? a.k : a.vp);
                src = p.in + s * p.in_seq + j * p.in_tok + h * p.in_head;
                to[it] = p.out + s * p.out_seq + j * p.out_tok + h * p.out_head;
            }
            x[it][0] = *(const uint2 *)(src + c0);
            x[it][1] = *(const uint2 *)(src + c1);
        }
    }
    if (tid < half) {
        const long long at = s * a.pos_seq + j * a.pos_tok;
        const double pos = a.pos64 ? (double)((const int64_t *)a.pos)[at] : (double)((const int32_t *)a.pos)[at];
        // the angle's turns: the product and 1 / 2 pi in two parts each, so that
        // what is left of positions of 2^50 turns is right to 2^-50
        const double f = (double)a.inv_freq[tid], k0 = 0x1.45f306dc9c883p-3, k1 = -0x1.6b01ec5417056p-57;
        const double angle = pos * f, angle1 = fma(pos, f, -angle);
        const double turns = angle * k0, turns1 = fma(angle, k0, -turns) + fma(angle, k1, angle1 * k0);
        float sn, cn;
        sincospif((float)(2.0 * ((turns - rint(turns)) + turns1)), &sn, &cn);
        cs[0][tid] = cn;
        cs[1][tid] = sn;
    }
    // (wa cos, wb sin, wb cos, wa sin) of the lane's pairs, for queries and keys
    float4 turn[2][4];
    const bool norm = a.qw != nullptr;
    uint2 wr[2][2];
    if (norm) {
        wr[0][0] = *(const uint2 *)(a.qw + c0);
        wr[0][1] = *(const uint2 *)(a.qw + c1);
        wr[1][0] = *(const uint2 *)(a.kw + c0);
        wr[1][1] = *(const uint2 *)(a.kw + c1);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float cn = turned ? cs[0][4 * l + i] : 1.0f, sn = turned ? cs[1][4 * l + i] : 0.0f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float2 w = norm ? pair_of<DT, INTER>(wr[k], i) : make_float2(1.0f, 1.0f);
            turn[k][i] = make_float4(w.x * cn, w.y * sn, w.y * cn, w.x * sn);
        }
    }
    auto rotate = [&](uint2 (&r)[2], const float4 (&m)[4]) {
        float2 f[4];
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = pair_of<DT, INTER>(r, i);
            ss = fmaf(f[i].x, f[i].x, fmaf(f[i].y, f[i].y, ss));
        }
        float inv = 1.0f;
        if (norm) {
            float mean = row_sum(ss) * (1.0f / D) + a.eps;
            // Squares out of fp32's range (bf16 rows only; a row's lanes agree): the
            // row is taken 2^80 times as large, or 2^-70.  One comparison of patterns.
            constexpr uint32_t least = 31u << 23, most = 255u << 23;           // 2^-96, infinity
            if (DT && __float_as_uint(mean) - least >= most - least) {
                const float by = mean < 1.0f ? 0x1p80f : 0x1p-70f;
                ss = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f[i].x *= by;
                    f[i].y *= by;
                    ss = fmaf(f[i].x, f[i].x, fmaf(f[i].y, f[i].y, ss));
                }
                mean = row_sum(ss) * (1.0f / D) + a.eps * by * by;
            }
            const bool tiny = !DT && mean < 0x1p-96f;      // (zeros and a tiny eps; the instruction takes no subnormal numbers)
            inv = __builtin_amdgcn_rsqf(tiny ? mean * 0x1p64f : mean) * (tiny ? 0x1p32f : 1.0f);
        } else if (!turned) {
            return;                                        // (as they came, whatever they are)
        }
        float u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] = fmaf(f[i].x, m[i].x, -(f[i].y * m[i].y)) * inv;
            v[i] = fmaf(f[i].y, m[i].z, f[i].x * m[i].w) * inv;
        }
        if (INTER) {
            r[0] = make_uint2(pack<DT>(u[0], v[0]), pack<DT>(u[1], v[1]));
            r[1] = make_uint2(pack<DT>(u[2], v[2]), pack<DT>(u[3], v[3]));
        } else {
            r[0] = make_uint2(pack<DT>(u[0], u[1]), pack<DT>(u[2], u[3]));
            r[1] = make_uint2(pack<DT>(v[0], v[1]), pack<DT>(v[2], v[3]));
        }
    };
#pragma unroll
    for (int it = 0; it < NR_AHEAD; ++it) {
        const int row = rw0 + it * NR_ROWS + g;
        if (it < rounds && row < nrows) {
            if (row < a.hq) rotate(x[it], turn[0]);
            else if (row < a.hq + a.hkv) rotate(x[it], turn[1]);
            // (streamed: 32768 tokens of 48 rows 130 us, 142 without)
            __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, x[it][0]), (uint64_t *)(to[it] + c0));
            __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, x[it][1]), (uint64_t *)(to[it] + c1));
        }
    }
}

}  // namespace

hipError_t launch_norm_rope(const NormRope &a, int dtype, int interleaved, hipStream_t s) {
    const int nrows = a.hq + a.hkv * (a.v ? 2 : 1), all = ceil_div(nrows, NR_ROWS);
    const long long tokens = (long long)a.seqs * a.n;
    // a token's rounds in one workgroup share its sines; with few tokens the
    // rounds go to workgroups of their own, as far as a grid's second dimension
    // goes.  us of captured calls, one round / up to four rounds a workgroup:
    //   tokens              16           256          512          1024         2048
    //   48 rows (32 + 16)   3.0 / 3.9    3.8 / 4.5    5.1 / 5.2    7.7 / 6.2    12.7 / 10.1
    //   80 rows (64 + 16)   3.0 / 4.3    4.7 / 5.1    7.0 / 5.8    11.2 / 8.5   23.8 / 18.0
    //   24 rows (16 + 8)    3.0 / 3.5    3.4 / 3.8    4.1 / 4.1    6.2 / 5.1    9.3 / 7.7
    const int rounds = tokens >= 512 || all > 65535 ? (all < NR_AHEAD ? all : NR_AHEAD) : 1;
    const dim3 grid((uint32_t)tokens, ceil_div(all, rounds));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, rounds); };
    if (dtype) {
        if (interleaved) go(k_norm_rope<1, true>); else go(k_norm_rope<1, false>);
    } else {
        if (interleaved) go(k_norm_rope<0, true>); else go(k_norm_rope<0, false>);
    }
    return hipGetLastError();
}

}  // namespace mosaic
