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
// A workgroup takes one token, 16 lanes a row: a lane's 16 bytes are 8
// channels, the sum of squares is four row rotations, and a lane's channels
// are the same in every row, so cos, sin and weights are read once for all of
// the token's rows.  64 lanes compute the token's sines and cosines.  HBM is
// the bound: every row is read and written once.
#include "mosaic_internal.h"

namespace mosaic {

namespace {

constexpr int NR_ROWS = 16;                                // rows of a workgroup's round

template <int ROR> __device__ __forceinline__ float row_ror_add(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + ROR, 0xf, 0xf, false));
}

// two of a lane's 8 channels from word i of its 16 bytes
template <int DT> __device__ __forceinline__ float2 unpack(uint32_t w) {
    return make_float2(h2f((uint16_t)w, DT), h2f((uint16_t)(w >> 16), DT));
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

// grid (tokens, rounds of a token's rows / rounds of a workgroup)
template <int DT, bool INTER>
__global__ void __launch_bounds__(256) k_norm_rope(NormRope a, int rounds) {
    __shared__ __align__(16) float cs[2][D / 2];
    const int tid = threadIdx.x, l = tid & 15, half = a.half;
    const long long t = blockIdx.x;
    const long long s = t / a.n, j = t - s * a.n;
    const int r0 = blockIdx.y * rounds;
    const int nrows = a.hq + 2 * a.hkv - (a.v ? 0 : a.hkv);
    if (tid < half) {
        const long long at = s * a.pos_seq + j * a.pos_tok;
        const double pos = a.pos64 ? (double)((const int64_t *)a.pos)[at] : (double)((const int32_t *)a.pos)[at];
        // the angle's turns: the product and 1 / 2 pi in two parts each, so that
        // what is left of positions of 2^50 turns is right to 2^-50
        const double f = (double)a.inv_freq[tid], c0 = 0x1.45f306dc9c883p-3, c1 = -0x1.6b01ec5417056p-57;
        const double angle = pos * f, angle1 = fma(pos, f, -angle);
        const double turns = angle * c0, turns1 = fma(angle, c0, -turns) + fma(angle, c1, angle1 * c0);
        float sn, cn;
        sincospif((float)(2.0 * ((turns - rint(turns)) + turns1)), &sn, &cn);
        cs[0][tid] = cn;
        cs[1][tid] = sn;
    }
    __syncthreads();
    const bool turned = 8 * l < 2 * half;
    // the lane's cosines and sines: channels c and c + half share one, or 2 i and 2 i + 1
    float cn[8], sn[8];
    const int i0 = INTER ? 4 * l : (8 * l < half ? 8 * l : 8 * l - half);
#pragma unroll
    for (int i = 0; i < (INTER ? 4 : 8); ++i) {
        cn[i] = turned ? cs[0][i0 + i] : 1.0f;
        sn[i] = turned ? cs[1][i0 + i] : 0.0f;
    }
    const bool low = 8 * l < half;                         // the lane holds the pairs' first channels
    const int partner = (tid & 48) + (turned ? (low ? l + half / 8 : l - half / 8) : l);
    for (int it = 0; it < rounds; ++it) {
        const int row = (r0 + it) * NR_ROWS + (tid >> 4);
        if (__all(row >= nrows)) break;
        const bool live = row < nrows;
        const int kind = row < a.hq ? 0 : (row < a.hq + a.hkv ? 1 : 2);
        const int h = kind == 0 ? row : (kind == 1 ? row - a.hq : row - a.hq - a.hkv);
        const NormRope::Part &p = kind == 0 ? a.q : (kind == 1 ? a.k : a.vp);
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (live) x = *(const uint4 *)(p.in + s * p.in_seq + j * p.in_tok + h * p.in_head + 8 * l);
        uint32_t o[4] = {x.x, x.y, x.z, x.w};
        uint32_t y[4];                                     // the partner channels, as they came
        if (!INTER)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (uint32_t)__shfl((int)o[i], partner, 64);
        if (live && kind < 2) {
            float f[8], g[8];
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 u = unpack<DT>(o[i]);
                f[2 * i] = u.x;
                f[2 * i + 1] = u.y;
                ss = fmaf(u.x, u.x, fmaf(u.y, u.y, ss));
                if (!INTER) {
                    const float2 v = unpack<DT>(y[i]);
                    g[2 * i] = v.x;
                    g[2 * i + 1] = v.y;
                }
            }
            const uint16_t *w = kind == 0 ? a.qw : a.kw;
            if (w) {
                ss = row_ror_add<8>(ss);
                ss = row_ror_add<4>(ss);
                ss = row_ror_add<2>(ss);
                ss = row_ror_add<1>(ss);
                const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
                const uint4 wm = *(const uint4 *)(w + 8 * l), wp = *(const uint4 *)(w + 8 * (partner & 15));
                const uint32_t m4[4] = {wm.x, wm.y, wm.z, wm.w}, p4[4] = {wp.x, wp.y, wp.z, wp.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 u = unpack<DT>(m4[i]);
                    f[2 * i] = f[2 * i] * r * u.x;
                    f[2 * i + 1] = f[2 * i + 1] * r * u.y;
                    if (!INTER) {
                        const float2 v = unpack<DT>(p4[i]);
                        g[2 * i] = g[2 * i] * r * v.x;
                        g[2 * i + 1] = g[2 * i + 1] * r * v.y;
                    }
                }
            }
            if (turned || w) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float u, v;
                    if (!turned) {
                        u = f[2 * i];
                        v = f[2 * i + 1];
                    } else if (INTER) {
                        u = fmaf(f[2 * i], cn[i], -(f[2 * i + 1] * sn[i]));
                        v = fmaf(f[2 * i + 1], cn[i], f[2 * i] * sn[i]);
                    } else {
                        const float s0 = low ? -sn[2 * i] : sn[2 * i], s1 = low ? -sn[2 * i + 1] : sn[2 * i + 1];
                        u = fmaf(f[2 * i], cn[2 * i], g[2 * i] * s0);
                        v = fmaf(f[2 * i + 1], cn[2 * i + 1], g[2 * i + 1] * s1);
                    }
                    o[i] = pack<DT>(u, v);
                }
            }
        }
        if (live) *(uint4 *)(p.out + s * p.out_seq + j * p.out_tok + h * p.out_head + 8 * l) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

}  // namespace

hipError_t launch_norm_rope(const NormRope &a, int dtype, int interleaved, hipStream_t s) {
    const int nrows = a.hq + a.hkv * (a.v ? 2 : 1), all = ceil_div(nrows, NR_ROWS);
    const long long tokens = (long long)a.seqs * a.n;
    // a token's rounds in one workgroup share its sines; with few tokens the
    // rounds go to workgroups of their own
    const int rounds = tokens >= 512 ? all : 1;
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
