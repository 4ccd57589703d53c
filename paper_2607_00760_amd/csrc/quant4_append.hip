// quant4_append.hip -- tokens into the 4-bit KV cache (mosaic_nibble_append).
//
// A row of a block gets a grid of 16 values: zero = its least value lo, scale =
// (hi - lo) / 15 rounded down to the element type, code = nearest((x - lo) /
// scale).  Rows are a channel's keys over the block's tokens (a head's strong
// channels are strong in every token, and would take the resolution of the
// others) and a token's values over the channels.  Differences are of halves,
// which no value of the type overflows.  A block is encoded once, when its last
// token arrives, from 16-bit tokens; until then its tokens wait in the tail, so
// the codes do not depend on how many calls brought the tokens.
//
// One workgroup per (block that the call may complete, pair): half of it takes
// the keys, half the values, a thread 4 tokens x 8 channels, 16 lanes a token.
// A token's least and largest value meet in its 16 lanes, a channel's in LDS,
// where one thread a channel makes the grid.  HBM is the bound: 512 bytes of a
// token are read, 128 and its share of the grids are written (4 x 32785 tokens of 8
// heads, 0.69 GB: 119 us, 5.8 TB/s).  One token of 8 or 64 sequences, 8 heads: 2.7
// and 3.6 us in a captured step, a launch and one chain of round trips.
#include <type_traits>

#include "quant4.h"

namespace mosaic {

namespace {

constexpr int QN4_ARRIVE = 32;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// 16-bit floating patterns as integers of the same order (and back), two in a word
typedef __attribute__((ext_vector_type(2))) short s16x2;
__device__ __forceinline__ s16x2 ordered(uint32_t w) {
    const s16x2 v = __builtin_bit_cast(s16x2, w);
    return v ^ ((v >> 15) & (short)0x7fff);
}
__device__ __forceinline__ s16x2 pk_max(s16x2 a, s16x2 b) { return __builtin_elementwise_max(a, b); }
// over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ s16x2 rows_max(s16x2 x) {
    uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    u = __builtin_bit_cast(uint32_t, pk_max(__builtin_bit_cast(s16x2, (uint32_t)a[0]), __builtin_bit_cast(s16x2, (uint32_t)a[1])));
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return pk_max(__builtin_bit_cast(s16x2, (uint32_t)b[0]), __builtin_bit_cast(s16x2, (uint32_t)b[1]));
}
// over the 16 lanes of a row
template <int ROR> __device__ __forceinline__ s16x2 ror_max(s16x2 x) {
    const int u = __builtin_bit_cast(int, x);
    return pk_max(x, __builtin_bit_cast(s16x2, __builtin_amdgcn_update_dpp(0, u, 0x120 + ROR, 0xf, 0xf, false)));
}
__device__ __forceinline__ s16x2 row_max(s16x2 x) { return ror_max<1>(ror_max<2>(ror_max<4>(ror_max<8>(x)))); }
// lane r of each four
template <int R> __device__ __forceinline__ float quad(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x55 * R, 0xf, 0xf, false));
}

struct Grid { uint32_t scale, zero; float inv, nl; };      // 16-bit patterns; 2 / scale, -lo / 2
// hi, lo: ordered patterns
template <int DT> __device__ __forceinline__ Grid grid_of(short hi, short lo) {
    const uint32_t both = __builtin_bit_cast(uint32_t, ordered(((uint32_t)(uint16_t)lo << 16) | (uint16_t)hi));
    const float h = h2f((uint16_t)both, DT), l = h2f((uint16_t)(both >> 16), DT);
    Grid g;
    g.nl = -0.5f * l;
    const float d = fmaf(h, 0.5f, g.nl), want = d / 7.5f;
    if (DT) {
        g.scale = __float_as_uint(want) >> 16;
    } else {
        const _Float16 n = (_Float16)want;
        g.scale = __builtin_bit_cast(uint16_t, n) - ((float)n > want ? 1u : 0u);
    }
    g.scale = max(g.scale, q4_least<DT>());
    g.zero = both >> 16;
    g.inv = 2.0f / h2f((uint16_t)g.scale, DT);
    if (!(d < INFINITY)) {                                 // a value that is not finite: the row stands for NaN
        g.scale = g.zero = DT ? 0x7fc0u : 0x7e00u;
        g.inv = 0.0f;
    }
    return g;
}
// 2^23 + code, as a pattern (a NaN's code is 0)
__device__ __forceinline__ uint32_t code_of(float x, float nl, float inv) {
    return __float_as_uint(__builtin_amdgcn_fmed3f(fmaf(x, 0.5f, nl) * inv, 0.0f, 15.0f) + 8388608.0f);
}

// grid (blocks that the call may complete, pairs).  The last of a pair's
// workgroups to have read the length writes the new one; grids of more than
// QN4_ARRIVE blocks leave that to a launch of its own.
template <int B, int DT>
__global__ void __launch_bounds__(8 * B) k_quant4_append(Q4Cache q, QNew nw) {
    constexpr int HW = 4 * B / 64;                         // waves of a half
    constexpr int VROW = B / 4 + 2;                        // a channel's codes, 4 a piece, and 4 bytes that part the banks
    __shared__ uint4 bnd[HW][16][2];                       // [wave][8 channels][largest, ~smallest], ordered
    __shared__ float2 grid[D];                             // (2 / scale, -lo / 2) of the channels
    __shared__ uint16_t vc[D][VROW];
    const int p = blockIdx.y, j = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = p / q.H, h = p - s * q.H;
    const int vals = tid >= 4 * B, ht = tid & (4 * B - 1);
    const int tg = ht >> 4, pc = ht & 15;
    // the thread's tokens: a quarter of the block apart for the keys (their rows
    // go out side by side), consecutive for the values (packed by token)
    const int t0 = vals ? 4 * tg : tg, step = vals ? 1 : B / 4;
    const int L = q.len(p);
    int n = nw.counts ? nw.counts[s] : nw.max_new;
    n = min(max(n, 0), nw.max_new);
    if (n == 0) return;
    if (n > q.cap - L) {                                   // no room: the sequence stays as it is
        if (j == 0 && h == 0 && tid == 0) q.refused[s] += 1;
        return;
    }
    const int f = L % B, first = L / B, done = (f + n) / B;
    int32_t *arrivals = q.arrivals + (uint64_t)p * Q_ARRIVALS;
    auto arrive = [&] {
        if (gridDim.x > QN4_ARRIVE) return;
        __syncthreads();                                   // every thread has read the length
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
        if (j * B >= f) {                                  // new tokens only
            const uint16_t *row = src + (int64_t)(j * B - f + t0) * tok + 8 * pc;
#pragma unroll
            for (int r = 0; r < 4; ++r) {                      // (streamed: 4 x 32785 tokens written and read back 257 us, 275 without)
                x[r] = __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4 *)row));
                row += step * tok;
            }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = t0 + step * r;               // token of the unfinished block and the new ones together
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
        const uint64_t blk = (uint64_t)p * q.N + first + j;
        if (!vals) {                                       // the channels' largest and smallest keys of the wave
            uint4 hl[2];
            uint32_t *o = (uint32_t *)hl;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                s16x2 hi = ordered(w[0][d]), lo = ~hi;
#pragma unroll
                for (int r = 1; r < 4; ++r) { hi = pk_max(hi, ordered(w[r][d])); lo = pk_max(lo, ~ordered(w[r][d])); }
                o[d] = __builtin_bit_cast(uint32_t, rows_max(hi));
                o[4 + d] = __builtin_bit_cast(uint32_t, rows_max(lo));
            }
            if (lane < 16) { bnd[wave][pc][0] = hl[0]; bnd[wave][pc][1] = hl[1]; }
        } else {
            s16x2 hl[4];                                   // (largest, ~smallest) of each token
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s16x2 hi = ordered(w[r][0]), lo = ~hi;
#pragma unroll
                for (int d = 1; d < 4; ++d) { hi = pk_max(hi, ordered(w[r][d])); lo = pk_max(lo, ~ordered(w[r][d])); }
                hl[r] = row_max(pk_max(s16x2{hi[0], lo[0]}, s16x2{hi[1], lo[1]}));
            }
            const int mine = lane & 3;                     // the token whose grid the lane makes
            const s16x2 m = mine < 2 ? (mine == 0 ? hl[0] : hl[1]) : (mine == 2 ? hl[2] : hl[3]);
            const Grid g = grid_of<DT>(m[0], (short)~m[1]);
            if (pc < 4) {
                uint16_t *vg = q.vg + blk * (2 * B) + t0 + pc;
                vg[0] = (uint16_t)g.scale;
                vg[B] = (uint16_t)g.zero;
            }
            const float inv[4] = {quad<0>(g.inv), quad<1>(g.inv), quad<2>(g.inv), quad<3>(g.inv)};
            const float nl[4] = {quad<0>(g.nl), quad<1>(g.nl), quad<2>(g.nl), quad<3>(g.nl)};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t c = 0;                            // (the patterns' 2^23 stays above the codes)
#pragma unroll
                for (int r = 3; r >= 0; --r) c = (c << 4) + code_of(half_of<DT>(w[r], i), nl[r], inv[r]);
                vc[8 * pc + i][tg] = (uint16_t)c;
            }
        }
        __syncthreads();
        if (tid < D) {                                     // the channels' grids
            short hi = -32768, lo = -32768;
#pragma unroll
            for (int i = 0; i < HW; ++i) {
                hi = max(hi, ((const short *)&bnd[i][tid >> 3][0])[tid & 7]);
                lo = max(lo, ((const short *)&bnd[i][tid >> 3][1])[tid & 7]);
            }
            const Grid g = grid_of<DT>(hi, (short)~lo);
            uint16_t *kg = q.kg + blk * (2 * D) + tid;
            kg[0] = (uint16_t)g.scale;
            kg[D] = (uint16_t)g.zero;
            grid[tid] = make_float2(g.inv, g.nl);
        }
        __syncthreads();
        if (!vals) {
            float2 g[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = grid[8 * pc + i];
            uint8_t *kp = q.k + blk * (B * D / 2) + 4 * pc;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t c = 0;
#pragma unroll
                for (int i = 7; i >= 0; --i) c = (c << 4) + code_of(half_of<DT>(w[r], i), g[i].y, g[i].x);
                // what the patterns' 2^23 have added up to: 0x4b000000 + (0x4b000000 << 4)
                *(uint32_t *)(kp + (t0 + step * r) * (D / 2)) = c - 0xfb000000u;
            }
        } else {                                           // 16 bytes of a channel's codes
            constexpr int PR = B / 32;                     // pieces of a channel
            const uint32_t *row = (const uint32_t *)&vc[ht / PR][8 * (ht % PR)];
            *(uint4 *)(q.v + blk * (B * D / 2) + 16 * ht) = make_uint4(row[0], row[1], row[2], row[3]);
        }
    }
    if (j > 0) { arrive(); return; }
    // the tokens that no block holds yet: from here on the tail's old rows have
    // been read (the barriers above), or stay where they are
    const int rest = f + n - done * B, from = done ? 0 : f;
    for (int i = tid; i < (rest - from) * 16; i += 8 * B) {
        const int t = from + (i >> 4), g = i & 15;
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

__global__ void __launch_bounds__(256) k_quant4_lens(Q4Cache q, QNew nw) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p >= q.S * q.H) return;
    const int L = q.len(p), n = min(max(nw.counts ? nw.counts[p / q.H] : nw.max_new, 0), nw.max_new);
    if (n <= q.cap - L) q.lens[p] = L + n;
}

}  // namespace

hipError_t launch_quant4_append(const Q4Cache &q, int block, int dtype, const QNew &n, hipStream_t s) {
    const int most = (int)(((long long)block - 1 + n.max_new) / block), pairs = q.S * q.H;
    const dim3 grid(most < 1 ? 1 : most, pairs);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(8 * block), 0, s, q, n); };
    if (block == 32) { if (dtype) go(k_quant4_append<32, 1>); else go(k_quant4_append<32, 0>); }
    else { if (dtype) go(k_quant4_append<64, 1>); else go(k_quant4_append<64, 0>); }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || most <= QN4_ARRIVE) return e;
    hipLaunchKernelGGL(k_quant4_lens, dim3(ceil_div(pairs, 256)), dim3(256), 0, s, q, n);
    return hipGetLastError();
}

}  // namespace mosaic
