// quant_append.hip -- tokens into the 8-bit KV cache (mosaic_quant_append).
//
// A block of B tokens of one (sequence, kv head) gets one scale for its keys
// and one for its values: a = max(max |x|, 2^-100), scale = a / Q, code =
// nearest(x * (Q / a)).  It is encoded once, when its last token arrives, from
// 16-bit tokens; until then its tokens wait in the tail, so the codes do not
// depend on how many calls brought the tokens.  A block's key bounds (per
// channel the largest and the smallest key, in units of a / 127, rounded
// outwards) come from the same registers.
//
// One workgroup per (block that the call may complete, pair): half of it takes
// the keys, half the values, a thread 4 tokens x 8 channels.  The values'
// codes are stored by channel, 4 x 4 bytes turned in registers.  HBM is the
// bound: 512 bytes of a token are read, 256 and the block's share are written.
#include <type_traits>

#include "quant.h"

namespace mosaic {

namespace {

constexpr int QN_ARRIVE = 32;

// bytes e of four words: the columns of a 4 x 4 byte matrix
__device__ __forceinline__ void turn4(const uint32_t (&r)[4], uint32_t (&c)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
    const uint32_t d = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), e = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
    c[0] = __builtin_amdgcn_perm(d, a, 0x05040100u);
    c[1] = __builtin_amdgcn_perm(d, a, 0x07060302u);
    c[2] = __builtin_amdgcn_perm(e, b, 0x05040100u);
    c[3] = __builtin_amdgcn_perm(e, b, 0x07060302u);
}

// 16-bit floating patterns as integers of the same order (and back), two in a
// word: the keys' bounds and both magnitudes are found without widening, half
// of the instructions (4 x 32785 tokens 158 -> 148 us)
typedef __attribute__((ext_vector_type(2))) short s16x2;
__device__ __forceinline__ s16x2 ordered(uint32_t w) {
    const s16x2 v = __builtin_bit_cast(s16x2, w);
    return v ^ ((v >> 15) & (short)0x7fff);
}
__device__ __forceinline__ s16x2 pk_max(s16x2 a, s16x2 b) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ s16x2 pk_min(s16x2 a, s16x2 b) { return __builtin_elementwise_min(a, b); }
__device__ __forceinline__ s16x2 word2(const uint4 &v, int d) {
    return __builtin_bit_cast(s16x2, ((const uint32_t *)&v)[d]);
}
// over the four lanes l, l ^ 16, l ^ 32, l ^ 48
template <typename F> __device__ __forceinline__ s16x2 rows_pk(s16x2 x, F f) {
    uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    u = __builtin_bit_cast(uint32_t, f(__builtin_bit_cast(s16x2, (uint32_t)a[0]), __builtin_bit_cast(s16x2, (uint32_t)a[1])));
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return f(__builtin_bit_cast(s16x2, (uint32_t)b[0]), __builtin_bit_cast(s16x2, (uint32_t)b[1]));
}

// Codes of four values already in units of the scale, one byte each.  No value
// of a block is past the largest code by more than a rounding, so nothing is
// clamped; integers come out of the lowest bits of 1.5 * 2^23 + y.
template <int FMT> __device__ __forceinline__ uint32_t codes4(const float (&y)[4]) {
    if (FMT == QF_E4M3) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    }
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(y[i] + 12582912.0f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u), __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), 0x05040100u);
}

// grid (blocks that the call may complete, pairs).  The last of a pair's
// workgroups to have read the length writes the new one; grids of more than
// QN_ARRIVE blocks leave that to a launch of its own (4 us): an arrival at one
// address takes 12 ns, and 1025 for each of 32 pairs take the prefill of 4 x
// 32785 tokens from 144 to 166 us (to 388 with the pairs' counters in one line).
template <int FMT, int B, int DT>
__global__ void __launch_bounds__(8 * B) k_quant_append(QCache q, QNew nw) {
    constexpr int HW = 4 * B / 64;                             // waves of a half
    __shared__ uint32_t red[2 * HW];
    __shared__ uint4 bnd[HW][16][2];                           // [wave][8 channels][upper, lower], ordered
    const int p = blockIdx.y, j = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = p / q.H, h = p - s * q.H;
    // 4 tokens x 8 channels of a thread: rows side by side for the keys, whose
    // codes lie by token, token groups side by side for the values
    const int vals = tid >= 4 * B, ht = tid & (4 * B - 1);
    const int t4 = vals ? ht & (B / 4 - 1) : ht >> 4, pc = vals ? ht / (B / 4) : ht & 15;
    const int L = q.len(p);
    int n = nw.counts ? nw.counts[s] : nw.max_new;
    n = min(max(n, 0), nw.max_new);
    if (n == 0) return;
    if (n > q.cap - L) {                                       // no room: the sequence stays as it is
        if (j == 0 && h == 0 && tid == 0) q.refused[s] += 1;
        return;
    }
    const int f = L % B, first = L / B, done = (f + n) / B;
    int32_t *arrivals = q.arrivals + (uint64_t)p * Q_ARRIVALS;
    auto arrive = [&] {
        if (gridDim.x > QN_ARRIVE) return;
        __syncthreads();                                       // every thread has read the length
        if (tid != 0) return;
        if (gridDim.x > 1) {
            if (__hip_atomic_fetch_add(arrivals, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != (int)gridDim.x - 1) return;
            __hip_atomic_store(arrivals, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        q.lens[p] = L + n;
    };
    if (j > 0 && j >= done) { arrive(); return; }
    const uint16_t *src = vals ? nw.v + s * nw.v_seq + h * nw.v_head : nw.k + s * nw.k_seq + h * nw.k_head;
    const int64_t tok = vals ? nw.v_tok : nw.k_tok;
    uint16_t *kt = q.kt + (uint64_t)p * B * D, *vt = q.vt + (uint64_t)p * B * D;
    if (j < done) {
        uint4 x[4];
        if (j * B >= f) {                                      // new tokens only
            const uint16_t *row = src + (int64_t)(j * B - f) * tok + (int64_t)(4 * t4) * tok + 8 * pc;
#pragma unroll
            for (int r = 0; r < 4; ++r) { x[r] = *(const uint4 *)row; row += tok; }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = 4 * t4 + r;                      // token of the unfinished block and the new ones together
                if (c >= f) x[r] = *(const uint4 *)(src + (int64_t)(c - f) * tok + 8 * pc);
                else if (!vals) x[r] = *(const uint4 *)(kt + c * D + 8 * pc);
                else {
                    uint16_t e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = vt[(8 * pc + i) * B + c];
                    __builtin_memcpy(&x[r], e, 16);
                }
            }
        }
        const uint32_t w[4][4] = {{x[0].x, x[0].y, x[0].z, x[0].w}, {x[1].x, x[1].y, x[1].z, x[1].w},
                                  {x[2].x, x[2].y, x[2].z, x[2].w}, {x[3].x, x[3].y, x[3].z, x[3].w}};
        s16x2 m = {0, 0};                                      // largest magnitudes, as 16-bit patterns
        if (!vals) {                                           // the channels' largest and smallest keys of the wave
            uint4 hl[2];
            uint32_t *o = (uint32_t *)hl;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const s16x2 k0 = ordered(w[0][d]), k1 = ordered(w[1][d]), k2 = ordered(w[2][d]), k3 = ordered(w[3][d]);
                const s16x2 hi = rows_pk(pk_max(pk_max(k0, k1), pk_max(k2, k3)), [](s16x2 u, s16x2 v) { return pk_max(u, v); });
                const s16x2 lo = rows_pk(pk_min(pk_min(k0, k1), pk_min(k2, k3)), [](s16x2 u, s16x2 v) { return pk_min(u, v); });
                m = pk_max(m, pk_max(hi, ~lo));                // (~ of a negative one is its magnitude)
                o[d] = __builtin_bit_cast(uint32_t, hi);
                o[4 + d] = __builtin_bit_cast(uint32_t, lo);
            }
            if (lane < 16) { bnd[wave][pc][0] = hl[0]; bnd[wave][pc][1] = hl[1]; }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int d = 0; d < 4; ++d) m = pk_max(m, __builtin_bit_cast(s16x2, w[r][d] & 0x7fff7fffu));
        }
        const uint32_t mw = wave_max_u((uint32_t)max((int)m[0], (int)m[1]));
        if (lane == 0) red[wave] = mw;
        __syncthreads();
        uint32_t mb = red[vals * HW];
#pragma unroll
        for (int i = 1; i < HW; ++i) mb = max(mb, red[vals * HW + i]);
        float a = h2f((uint16_t)mb, DT);
        a = a < QLEAST ? QLEAST : a;                           // (a NaN stays one)
        const float inv = q_top(FMT) / a;
        const uint64_t blk = (uint64_t)p * q.N + first + j;
        if (tid == 4 * B) q.vs[blk] = a / q_top(FMT);
        if (tid == 0) { q.ks[blk] = a / q_top(FMT); q.bs[blk] = a / 127.0f; }
        uint32_t c[4][2];                                      // [token][channels 0..3, 4..7]
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float z[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = w[r][2 * e + (i >> 1)];
                    z[i] = h2f((uint16_t)((i & 1) ? (u >> 16) : u), DT) * inv;
                }
                c[r][e] = codes4<FMT>(z);
            }
        if (!vals) {
            uint8_t *kp = q.k + blk * (B * D);
#pragma unroll
            for (int r = 0; r < 4; ++r)                        // (streamed: 148 -> 145 us; the values' 4-byte pieces gain nothing)
                __builtin_nontemporal_store((uint64_t)c[r][1] << 32 | c[r][0], (uint64_t *)(kp + (4 * t4 + r) * D + 8 * pc));
            if (tid < D / 2) {                                 // two channels each
                const float unit = 127.0f / a;
                const int g = tid >> 2, d = tid & 3;
                s16x2 hi = word2(bnd[0][g][0], d), lo = word2(bnd[0][g][1], d);
#pragma unroll
                for (int i = 1; i < HW; ++i) { hi = pk_max(hi, word2(bnd[i][g][0], d)); lo = pk_min(lo, word2(bnd[i][g][1], d)); }
                const uint32_t hb = __builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, hi)));
                const uint32_t lb = __builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, lo)));
                uint32_t up = 0, down = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float u = ceilf(h2f((uint16_t)(hb >> (16 * i)), DT) * unit), l = floorf(h2f((uint16_t)(lb >> (16 * i)), DT) * unit);
                    up |= ((uint32_t)(int)__builtin_amdgcn_fmed3f(u, -127.0f, 127.0f) & 0xffu) << (8 * i);
                    down |= ((uint32_t)(int)__builtin_amdgcn_fmed3f(l, -127.0f, 127.0f) & 0xffu) << (8 * i);
                }
                uint16_t *bp = (uint16_t *)(q.bounds + blk * (2 * D));
                bp[tid] = (uint16_t)up;
                bp[D / 2 + tid] = (uint16_t)down;
            }
        } else {
            uint8_t *vp = q.v + blk * (B * D) + 4 * t4;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t r[4] = {c[0][e], c[1][e], c[2][e], c[3][e]};
                uint32_t o[4];
                turn4(r, o);
#pragma unroll
                for (int i = 0; i < 4; ++i) *(uint32_t *)(vp + (8 * pc + 4 * e + i) * B) = o[i];
            }
        }
    }
    if (j > 0) { arrive(); return; }
    // the tokens that no block holds yet: from here on the tail's old rows have
    // been read (the barrier above), or stay where they are
    const int rest = f + n - done * B, t0 = done ? 0 : f;
    for (int i = tid; i < (rest - t0) * 16; i += 8 * B) {
        const int t = t0 + (i >> 4), g = i & 15;
        const int64_t at = (int64_t)(done * B + t - f);
        const uint4 kx = *(const uint4 *)(nw.k + s * nw.k_seq + h * nw.k_head + at * nw.k_tok + 8 * g);
        const uint4 vx = *(const uint4 *)(nw.v + s * nw.v_seq + h * nw.v_head + at * nw.v_tok + 8 * g);
        *(uint4 *)(kt + t * D + 8 * g) = kx;
        const uint32_t w[4] = {vx.x, vx.y, vx.z, vx.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) vt[(8 * g + e) * B + t] = (uint16_t)((e & 1) ? (w[e >> 1] >> 16) : w[e >> 1]);
    }
    arrive();
}

__global__ void __launch_bounds__(256) k_quant_lens(QCache q, QNew nw) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p >= q.S * q.H) return;
    const int L = q.len(p), n = min(max(nw.counts ? nw.counts[p / q.H] : nw.max_new, 0), nw.max_new);
    if (n <= q.cap - L) q.lens[p] = L + n;
}

}  // namespace

hipError_t launch_quant_append(const QCache &q, int fmt, int block, int dtype, const QNew &n, hipStream_t s) {
    const int most = (block - 1 + n.max_new) / block, pairs = q.S * q.H;
    const dim3 grid(most < 1 ? 1 : most, pairs);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(8 * block), 0, s, q, n); };
    auto by_type = [&](auto f, auto b) {
        constexpr int F = decltype(f)::value, B = decltype(b)::value;
        if (dtype) go(k_quant_append<F, B, 1>); else go(k_quant_append<F, B, 0>);
    };
    using std::integral_constant;
    if (fmt == QF_INT8) {
        if (block == 32) by_type(integral_constant<int, QF_INT8>{}, integral_constant<int, 32>{});
        else by_type(integral_constant<int, QF_INT8>{}, integral_constant<int, 64>{});
    } else {
        if (block == 32) by_type(integral_constant<int, QF_E4M3>{}, integral_constant<int, 32>{});
        else by_type(integral_constant<int, QF_E4M3>{}, integral_constant<int, 64>{});
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || most <= QN_ARRIVE) return e;
    hipLaunchKernelGGL(k_quant_lens, dim3(ceil_div(pairs, 256)), dim3(256), 0, s, q, n);
    return hipGetLastError();
}

}  // namespace mosaic
