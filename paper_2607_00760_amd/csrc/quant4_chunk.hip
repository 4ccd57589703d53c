// quant4_chunk.hip -- attention of several query tokens of a sequence over the
// 4-bit KV cache (mosaic_nibble_attend): chunks of a prompt, drafted tokens,
// queries that look at an encoder's states.
//
// K and V are what the cache reads back, zero + scale * code rounded to the
// element type, so one value serves every query.  A pair's queries are rows
// (token, head of the group); a workgroup takes 32 RW of them and walks the
// tokens 64 at a time, each 64 worked out once into LDS for all of its waves:
// keys by token, values by channel.  A wave holds 32 rows: S^T = K Q^T, the
// softmax with running maximum and sum, O^T += V^T P^T.  With that side of the
// products a row's logits lie in two lanes, and, the tokens dealt to the first
// product's rows as the second one asks for them, its weights go into the
// second product without leaving their lanes.
//
// Rows are many or few: with RW = 4 four waves share 64 tokens; with RW = 1
// each takes 64 tokens of its own and they are joined at the end.  Where there
// are too few rows for the chip the tokens are split over workgroups, which
// k_chunk_join joins.
#include <type_traits>

#include "quant4.h"

namespace mosaic {

namespace {

constexpr int CK_TILE = 64;                                // tokens of a step
constexpr int CK_WAVES = 4;
constexpr int CK_SLOTS = 512;                              // workgroups that take part in splits, at most
constexpr int CK_ROWS = 128;                               // rows of a workgroup at most

// Weights are this power of two times as large: as fp16 numbers those of 2^-25
// and less of the row's largest would vanish, and a million of them count.
template <int DT> constexpr float CK_POW = DT ? 0.0f : 14.0f;

typedef __attribute__((ext_vector_type(16))) float cf16;
template <int DT> __device__ __forceinline__ cf16 mma32(uint4 a, uint4 b, cf16 c) {
    if constexpr (DT) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(dbf8, a), __builtin_bit_cast(dbf8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(dhf8, a), __builtin_bit_cast(dhf8, b), c, 0, 0, 0);
}

// over lanes l and l ^ 32
template <typename F> __device__ __forceinline__ float halves(float x, F f) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return f(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// zero + scale * code of eight codes, rounded
template <int DT> __device__ __forceinline__ uint4 values8(uint32_t c, const float (&s)[8], const float (&z)[8]) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(s[i], (float)((c >> (4 * i)) & 15u), z[i]);
    return make_uint4(pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]), pack16<DT>(x[4], x[5]), pack16<DT>(x[6], x[7]));
}
template <int DT> __device__ __forceinline__ void widen8(uint4 w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = half_of<DT>(u, i);
}

// a row tile's share of the work, the same in the attention and in the join
struct ChunkPlan {
    int p, s, h, row0;                                     // pair, its sequence and kv head, the tile's first row
    int L, m, nt, per, used;                               // tokens, queries, steps of 64, of a split, splits with any
};
__device__ __forceinline__ ChunkPlan chunk_plan(const Q4Cache &q, const QChunk &c, int id, int tiles, int rows, int ns) {
    ChunkPlan r;
    const int pairs = q.S * q.H, t = tiles - 1 - id / pairs;       // (a pair's last tiles see most: first; one XCD's, if H is 8)
    r.p = id % pairs;
    r.s = r.p / q.H;
    r.h = r.p - r.s * q.H;
    r.row0 = t * rows;
    r.L = q.len(r.p);
    r.m = min(max(c.counts ? c.counts[r.s] : c.n, 0), c.n);
    const int last = min(r.m - 1, (r.row0 + rows - 1) / q.G);      // the tile's last query
    const int seen = r.row0 >= r.m * q.G ? 0 : max(c.causal ? r.L - r.m + last + 1 : r.L, 0);
    r.nt = (seen + CK_TILE - 1) / CK_TILE;
    r.per = (r.nt + ns - 1) / ns;
    r.used = r.per ? (r.nt + r.per - 1) / r.per : 0;
    return r;
}

template <int B, int DT, int RW>
__global__ void __launch_bounds__(64 * CK_WAVES)
k_chunk(Q4Cache q, QChunk c, int tiles, int ns, float *part) {
    constexpr int TW = CK_WAVES / RW, GT = 64 * RW;        // groups of waves with a step of their own, threads of a group
    constexpr int KR = GT / 16, KP = CK_TILE / KR;         // keys: tokens of a pass, passes
    constexpr int VR = GT / 8, VP = D / VR;                // values: channels of a pass, passes
    constexpr int NB = CK_TILE / B;                        // blocks of a step
    __shared__ __align__(16) uint8_t lds[TW][2 * CK_TILE * D * 2];
    __shared__ float ml[CK_WAVES][32][2];
    const int id = blockIdx.x / ns, split = blockIdx.x - id * ns;
    const ChunkPlan pl = chunk_plan(q, c, id, tiles, 32 * RW, ns);
    if (pl.row0 >= pl.m * q.G) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tw = wave / RW, rw = wave % RW, gt = tid & (GT - 1);
    const int t0 = split * pl.per, t1 = min(pl.nt, t0 + pl.per);
    if (split > 0 && t0 >= t1) return;                     // (split 0 writes what nothing is seen of, too)
    uint8_t *kl = lds[tw], *vl = lds[tw] + CK_TILE * D * 2;
    const int l32 = lane & 31, hl = lane >> 5;
    const int row = pl.row0 + 32 * rw + l32, qi = row / q.G, head = pl.h * q.G + row - qi * q.G;
    const bool valid = qi < pl.m;
    const int seen = valid ? (c.causal ? pl.L - pl.m + qi + 1 : pl.L) : 0;     // tokens that the row attends
    const int all = c.causal ? pl.L - pl.m + pl.row0 / q.G + 1 : pl.L;         // that every row of the workgroup does
    const float zs = fabsf(c.scale) * 1.44269504088896340736f;
    uint4 qf[8];                                           // channels 16 e + 8 hl + [0, 8) of the row
    {
        const uint16_t *qp = c.q + pl.s * c.q_seq + qi * c.q_tok + head * c.q_head + 8 * hl;
        const uint32_t flip = c.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            qf[e] = valid ? *(const uint4 *)(qp + 16 * e) : make_uint4(0, 0, 0, 0);
            qf[e].x ^= flip; qf[e].y ^= flip; qf[e].z ^= flip; qf[e].w ^= flip;
        }
    }
    // keys: tokens kt0 + KR i, channels 8 kc + [0, 8); values: channels vc0 + VR i, tokens 8 vo + [0, 8)
    const int kt0 = gt >> 4, kc = gt & 15, vc0 = gt >> 3, vo = gt & 7;
    const int whole = pl.L / B, tail = pl.L % B;
    const uint64_t pb = (uint64_t)pl.p * q.N;
    uint32_t kq[KP], vq[VP];
    uint4 kg[NB][2], vg[2];
    auto load = [&](int t) {                               // the step's codes and grids (blocks that are whole)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (NB * t + b >= whole) continue;
            const uint64_t blk = pb + (uint32_t)(NB * t + b);
            const uint16_t *g = q.kg + blk * (2 * D) + 8 * kc;
            kg[b][0] = *(const uint4 *)g;
            kg[b][1] = *(const uint4 *)(g + D);
        }
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int tk = kt0 + KR * i, b = NB * t + tk / B;
            if (b < whole) kq[i] = *(const uint32_t *)(q.k + (pb + (uint32_t)b) * (B * D / 2) + (tk % B) * (D / 2) + 4 * kc);
        }
        const int b = NB * t + 8 * vo / B, at = 8 * vo % B;
        if (b < whole) {
            const uint64_t blk = pb + (uint32_t)b;
            vg[0] = *(const uint4 *)(q.vg + blk * (2 * B) + at);
            vg[1] = *(const uint4 *)(q.vg + blk * (2 * B) + B + at);
#pragma unroll
            for (int i = 0; i < VP; ++i) vq[i] = *(const uint32_t *)(q.v + blk * (B * D / 2) + (vc0 + VR * i) * (B / 2) + at / 2);
        }
    };
    auto k_at = [&](int t, int piece) { return (uint4 *)(kl + t * 256 + 16 * (piece ^ (t & 15))); };
    auto v_at = [&](int ch, int piece) { return (uint4 *)(vl + ch * 128 + 16 * (piece ^ ((ch >> 1) & 7))); };
    auto store = [&](int t) {                              // into LDS; tokens past the last are zeros
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int tk = kt0 + KR * i, bi = tk / B, b = NB * t + bi;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (b < whole) {
                float s[8], z[8];
                widen8<DT>(kg[bi][0], s);
                widen8<DT>(kg[bi][1], z);
                x = values8<DT>(kq[i], s, z);
            } else if (b == whole && tk % B < tail) {
                x = *(const uint4 *)(q.kt + ((uint64_t)pl.p * B + tk % B) * D + 8 * kc);
            }
            *k_at(tk, kc) = x;
        }
        const int b = NB * t + 8 * vo / B, at = 8 * vo % B;
        float s[8], z[8];
        widen8<DT>(vg[0], s);
        widen8<DT>(vg[1], z);
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            const int ch = vc0 + VR * i;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (b < whole) {
                x = values8<DT>(vq[i], s, z);
            } else if (b == whole) {
                const int keep = tail - at;                // tokens of the eight
                if (keep > 0) x = *(const uint4 *)(q.vt + ((uint64_t)pl.p * D + ch) * B + at);
                x.x = keep >= 2 ? x.x : (keep == 1 ? x.x & 0xffffu : 0u);
                x.y = keep >= 4 ? x.y : (keep == 3 ? x.y & 0xffffu : 0u);
                x.z = keep >= 6 ? x.z : (keep == 5 ? x.z & 0xffffu : 0u);
                x.w = keep >= 8 ? x.w : (keep == 7 ? x.w & 0xffffu : 0u);
            }
            *v_at(ch, vo) = x;
        }
    };
    cf16 acc[4];                                           // [32 channels][8 (i / 4) + 4 hl + i % 4], the lane's row
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[ct][i] = 0.0f;
    float m_run = -INFINITY, l_run = 0.0f;
    // row r of the first product is the step's token (r & 16) + 8 (r / 4 & 1) + 4 (r / 8 & 1) + r % 4
    const int tau = (l32 & 16) + 8 * ((l32 >> 2) & 1) + 4 * ((l32 >> 3) & 1) + (l32 & 3);
    const int turns = (t1 - t0 + TW - 1) / TW;
    if (t0 + tw < t1) load(t0 + tw);
    for (int u = 0; u < turns; ++u) {
        const int t = t0 + u * TW + tw;
        lds_barrier();                                     // the last step has been read
        if (t < t1) store(t);
        if (t + TW < t1) load(t + TW);
        lds_barrier();
        if (t >= t1) continue;
        cf16 z[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[n][i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[n] = mma32<DT>(*k_at(32 * n + tau, 2 * e + hl), qf[e], z[n]);
        }
        // z[n][i]: token 64 t + 32 n + 16 (i / 8) + 8 hl + i % 8
        if (CK_TILE * (t + 1) > all) {                     // some row does not see all of them
            const int left = seen - (CK_TILE * t + 8 * hl);
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * n + 16 * (i >> 3) + (i & 7) >= left) z[n][i] = -INFINITY;
        }
        float cm = -INFINITY;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) cm = fmaxf(cm, z[n][i]);
        cm = halves(cm, [](float a, float b) { return fmaxf(a, b); });
        const float mn = fmaxf(m_run, cm), mb = mn == -INFINITY ? 0.0f : mn;
        const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - mb) * zs);
        m_run = mn;
        l_run *= alpha;
        uint4 pf[4];                                       // weights of tokens 16 e + 8 hl + [0, 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = z[e >> 1][8 * (e & 1) + i];
                x[i] = d == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(fmaf(d - mb, zs, CK_POW<DT>));
                l_run += x[i];
            }
            pf[e] = make_uint4(pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]), pack16<DT>(x[4], x[5]), pack16<DT>(x[6], x[7]));
        }
        if (!__all(alpha == 1.0f)) {
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[ct][i] *= alpha;
        }
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[ct] = mma32<DT>(*v_at(32 * ct + l32, 2 * e + hl), pf[e], acc[ct]);
    }
    l_run = halves(l_run, [](float a, float b) { return a + b; });
    if (TW > 1) {                                          // the waves joined, each a quarter of the channels
        __syncthreads();
        float *mine = (float *)lds[0];                     // [wave][channel][row]: 64 KB of 128
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(wave * D + 32 * ct + 8 * (i >> 2) + 4 * hl + (i & 3)) * 32 + l32] = acc[ct][i];
        if (hl == 0) { ml[wave][l32][0] = m_run; ml[wave][l32][1] = l_run; }
        __syncthreads();
        float m[CK_WAVES], f[CK_WAVES];
        m_run = -INFINITY;
#pragma unroll
        for (int w = 0; w < CK_WAVES; ++w) { m[w] = ml[w][l32][0]; m_run = fmaxf(m_run, m[w]); }
        l_run = 0.0f;
#pragma unroll
        for (int w = 0; w < CK_WAVES; ++w) {
            f[w] = m[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m[w] - m_run) * zs);
            l_run += f[w] * ml[w][l32][1];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {                     // channels 32 wave + 8 (i / 4) + 4 hl + i % 4
            float a = 0.0f;
#pragma unroll
            for (int w = 0; w < CK_WAVES; ++w) a += f[w] * mine[(w * D + 32 * wave + 8 * (i >> 2) + 4 * hl + (i & 3)) * 32 + l32];
            acc[0][i] = a;
        }
    }
    const float inv = l_run > 0.0f ? 1.0f / l_run : (l_run != l_run ? l_run : 0.0f);
    const int ch0 = TW > 1 ? 32 * wave : 0;
    if (pl.used <= 1) {
        if (!valid) return;
        uint16_t *op = c.out + pl.s * c.o_seq + qi * c.o_tok + head * c.o_head + ch0 + 4 * hl;
#pragma unroll
        for (int ct = 0; ct < (TW > 1 ? 1 : 4); ++ct)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(uint2 *)(op + 32 * ct + 8 * a) = make_uint2(pack16<DT>(acc[ct][4 * a] * inv, acc[ct][4 * a + 1] * inv),
                                                              pack16<DT>(acc[ct][4 * a + 2] * inv, acc[ct][4 * a + 3] * inv));
        return;
    }
    // a split's averages, and (maximum, sum)
    float *to = part + (uint64_t)blockIdx.x * (32 * RW) * (D + 4) + (row - pl.row0) * (D + 4);
    if (hl == 0 && (TW == 1 || wave == 0)) *(float2 *)to = make_float2(m_run == -INFINITY ? m_run : m_run * zs, l_run);
#pragma unroll
    for (int ct = 0; ct < (TW > 1 ? 1 : 4); ++ct)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *(float4 *)(to + 4 + ch0 + 32 * ct + 8 * a + 4 * hl) = make_float4(acc[ct][4 * a] * inv, acc[ct][4 * a + 1] * inv, acc[ct][4 * a + 2] * inv,
                                                                               acc[ct][4 * a + 3] * inv);
}

// the splits of a row tile joined, in their order; grid (row tiles and pairs, rows / 8), 32 lanes a row
template <int DT>
__global__ void __launch_bounds__(256) k_chunk_join(Q4Cache q, QChunk c, int tiles, int rows, int ns, const float *part) {
    const ChunkPlan pl = chunk_plan(q, c, blockIdx.x, tiles, rows, ns);
    if (pl.used <= 1) return;
    const int r = 8 * blockIdx.y + (threadIdx.x >> 5), ch = 4 * (threadIdx.x & 31);
    const int row = pl.row0 + r, qi = row / q.G, head = pl.h * q.G + row - qi * q.G;
    if (qi >= pl.m) return;
    const float *from = part + (uint64_t)blockIdx.x * ns * rows * (D + 4) + r * (D + 4);
    float M = -INFINITY, S = 0.0f;
    float4 A = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < pl.used; ++k) {
        const float *o = from + (uint64_t)k * rows * (D + 4);
        const float2 x = *(const float2 *)o;
        const float4 a = *(const float4 *)(o + 4 + ch);
        const float mn = fmaxf(M, x.x), mb = mn == -INFINITY ? 0.0f : mn;
        float f = S * __builtin_amdgcn_exp2f(M - mb), g = x.y * __builtin_amdgcn_exp2f(x.x - mb);
        S = f + g;
        const float inv = S > 0.0f ? 1.0f / S : (S != S ? S : 0.0f);
        f *= inv;
        g *= inv;
        A = make_float4(A.x * f + a.x * g, A.y * f + a.y * g, A.z * f + a.z * g, A.w * f + a.w * g);
        M = mn;
    }
    *(uint2 *)(c.out + pl.s * c.o_seq + qi * c.o_tok + head * c.o_head + ch) = make_uint2(pack16<DT>(A.x, A.y), pack16<DT>(A.z, A.w));
}

}  // namespace

size_t quant4_chunk_ws_bytes() { return (size_t)CK_SLOTS * CK_ROWS * (D + 4) * sizeof(float); }

hipError_t launch_quant4_chunk(const Q4Cache &q, int block, int dtype, const QChunk &c, float *part, hipStream_t s) {
    const int pairs = q.S * q.H, all = c.n * q.G;
    const int rows = all <= 32 ? 32 : CK_ROWS, tiles = (all + rows - 1) / rows;
    const long long wgs = (long long)pairs * tiles;
    const int most = ceil_div(q.cap, 4 * CK_TILE);         // (four steps a split at least)
    int ns = (int)(CK_SLOTS / wgs);
    ns = ns < 1 ? 1 : (ns > most ? most : ns);
    const dim3 grid((uint32_t)(wgs * ns));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * CK_WAVES), 0, s, q, c, tiles, ns, part); };
    auto by_rows = [&](auto b, auto dt) {
        constexpr int BL = decltype(b)::value, T = decltype(dt)::value;
        if (rows == 32) go(k_chunk<BL, T, 1>); else go(k_chunk<BL, T, 4>);
    };
    auto by_type = [&](auto b) { if (dtype) by_rows(b, std::integral_constant<int, 1>{}); else by_rows(b, std::integral_constant<int, 0>{}); };
    if (block == 32) by_type(std::integral_constant<int, 32>{}); else by_type(std::integral_constant<int, 64>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || ns == 1) return e;
    const dim3 jgrid((uint32_t)wgs, rows / 8);
    if (dtype) hipLaunchKernelGGL(k_chunk_join<1>, jgrid, dim3(256), 0, s, q, c, tiles, rows, ns, part);
    else hipLaunchKernelGGL(k_chunk_join<0>, jgrid, dim3(256), 0, s, q, c, tiles, rows, ns, part);
    return hipGetLastError();
}

}  // namespace mosaic
