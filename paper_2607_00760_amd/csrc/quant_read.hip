// quant_read.hip -- a run of each sequence's tokens out of the 4-bit and the
// 8-bit KV cache, as 16-bit rows (mosaic_nibble_read, mosaic_quant_read).
//
// A code's value is worked out in fp32 (zero + scale * code, or scale * code)
// and rounded once to the element type; the unfinished block's tokens are
// copied.  One workgroup per (block of the cache that the run may touch, pair).
// Keys lie by token and go straight through; values lie by channel and are
// turned through LDS: a thread takes 4 tokens x 8 channels, 16 lanes a row of
// the output.  Rows before the first token and past the last are not written.
// HBM is the bound: codes are read once, 512 bytes of a token are written (8 x 32 K
// tokens of 8 heads out of 4 bits, 1.37 GB: 240 us, 5.7 TB/s; a copy reaches 4.95.
// The last 5001 of 16 ragged sequences of 4 heads out of E4M3: 45 us, 5.4 TB/s).
#include <type_traits>

#include "quant4.h"

namespace mosaic {

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int QR_INT4 = 2;                                 // beside QF_E4M3 and QF_INT8

// code i of a word as a number
template <int FMT> __device__ __forceinline__ float code4(uint32_t w, int i) {
    if (FMT == QF_INT8) return (float)(int8_t)(w >> (8 * i));
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return i < 2 ? lo[i & 1] : hi[i & 1];
}
__device__ __forceinline__ float nibble(uint32_t w, int i) { return (float)((w >> (4 * i)) & 15u); }

template <int FMT, int B, int DT, typename C>
__global__ void __launch_bounds__(256) k_quant_read(C q, QOut o) {
    constexpr bool I4 = FMT == QR_INT4;
    constexpr int VB = I4 ? B / 2 : B;                     // bytes of a channel's values
    __shared__ uint32_t vc[D][VB / 4 + 1];                 // (the odd word parts the banks)
    const int p = blockIdx.y, tid = threadIdx.x, tg = tid >> 4, pc = tid & 15;
    const int s = p / q.H, h = p - s * q.H;
    const int L = q.len(p);
    const int64_t start = o.starts ? o.starts[s] : o.start, end = min(start + o.n, (int64_t)L);
    const int64_t from = max(start, (int64_t)0);
    const int64_t b = from / B + blockIdx.x;
    if (b * B >= end) return;
    const int first = (int)(b * B), whole = L / B;
    uint16_t *ko = o.k + s * o.k_seq + h * o.k_head + 8 * pc, *vo = o.v + s * o.v_seq + h * o.v_head + 8 * pc;
    auto held = [&](int t) { return t >= from && t < end; };
    auto put = [&](uint16_t *base, int64_t tok, int t, uint4 x) {
        // (streamed: 4 x 32785 tokens of 8 heads written and read back 211 us, 256 with plain stores;
        // the codes, which a cache that was just written still holds, are not: 224)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (u32x4 *)(base + (t - start) * tok));
    };
    if (b >= whole) {                                      // the unfinished block
        const uint16_t *kt = q.kt + (uint64_t)p * B * D + 8 * pc, *vt = q.vt + (uint64_t)p * B * D + 8 * pc * B;
#pragma unroll
        for (int i = 0; i < B / 16; ++i) {
            const int t = 16 * i + tg;
            if (!held(first + t)) continue;
            put(ko, o.k_tok, first + t, *(const uint4 *)(kt + t * D));
            uint32_t e[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) e[c] = vt[(2 * c) * B + t] | (uint32_t)vt[(2 * c + 1) * B + t] << 16;
            put(vo, o.v_tok, first + t, make_uint4(e[0], e[1], e[2], e[3]));
        }
        return;
    }
    const uint64_t blk = (uint64_t)p * q.N + (uint64_t)b;
    const uint8_t *kp = q.k + blk * (B * D * (I4 ? 1 : 2) / 2), *vp = q.v + blk * (D * VB);
    for (int i = tid; i < D * VB / 16; i += 256) {
        const uint4 x = *(const uint4 *)(vp + 16 * i);
        uint32_t *to = &vc[16 * i / VB][(16 * i % VB) / 4];
        to[0] = x.x; to[1] = x.y; to[2] = x.z; to[3] = x.w;
    }
    float ks[8], kz[8];
    if constexpr (I4) {
        const uint16_t *kg = q.kg + blk * (2 * D) + 8 * pc;
        const uint4 a = *(const uint4 *)kg, z = *(const uint4 *)(kg + D);
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, zw[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { ks[i] = half_of<DT>(aw, i); kz[i] = half_of<DT>(zw, i); }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) ks[i] = q.ks[blk];
    }
#pragma unroll
    for (int i = 0; i < B / 16; ++i) {
        const int t = 16 * i + tg;
        if (!held(first + t)) continue;
        float x[8];
        if constexpr (I4) {
            const uint32_t c = *(const uint32_t *)(kp + t * (D / 2) + 4 * pc);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf(ks[e], nibble(c, e), kz[e]);
        } else {
            const uint2 c = *(const uint2 *)(kp + t * D + 8 * pc);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = ks[e] * code4<FMT>(e < 4 ? c.x : c.y, e & 3);
        }
        put(ko, o.k_tok, first + t, make_uint4(pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]), pack16<DT>(x[4], x[5]), pack16<DT>(x[6], x[7])));
    }
    __syncthreads();
    if (4 * tg >= B) return;
    uint32_t c[8];                                         // codes of tokens 4 tg + [0, 4), a channel each
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = I4 ? ((const uint16_t *)vc[8 * pc + i])[tg] : vc[8 * pc + i][tg];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int t = 4 * tg + r;
        if (!held(first + t)) continue;
        float x[8];
        if constexpr (I4) {
            const uint16_t *vg = q.vg + blk * (2 * B) + t;
            const float vs = h2f(vg[0], DT), vz = h2f(vg[B], DT);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf(vs, nibble(c[e], r), vz);
        } else {
            const float vs = q.vs[blk];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = vs * code4<FMT>(c[e], r);
        }
        put(vo, o.v_tok, first + t, make_uint4(pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]), pack16<DT>(x[4], x[5]), pack16<DT>(x[6], x[7])));
    }
}

template <int FMT, typename C> hipError_t launch_read(const C &q, int block, int dtype, const QOut &o, hipStream_t s) {
    // blocks that n tokens touch, wherever they start; the cache has no more
    const long long most = ((long long)o.n + block - 2) / block + 1;
    const dim3 grid((uint32_t)(most < q.N ? most : q.N), q.S * q.H);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, q, o); };
    if (block == 32) { if (dtype) go(k_quant_read<FMT, 32, 1, C>); else go(k_quant_read<FMT, 32, 0, C>); }
    else { if (dtype) go(k_quant_read<FMT, 64, 1, C>); else go(k_quant_read<FMT, 64, 0, C>); }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quant4_read(const Q4Cache &q, int block, int dtype, const QOut &o, hipStream_t s) {
    return launch_read<QR_INT4>(q, block, dtype, o, s);
}
hipError_t launch_quant_read(const QCache &q, int fmt, int block, int dtype, const QOut &o, hipStream_t s) {
    return fmt == QF_INT8 ? launch_read<QF_INT8>(q, block, dtype, o, s) : launch_read<QF_E4M3>(q, block, dtype, o, s);
}

}  // namespace mosaic
