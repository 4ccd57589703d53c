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
// second product without leaving their lanes, rounded to the element type: each
// is off by half a step at most, as much as the output's own rounding.
//
// What bounds it.  Many rows: 2048 queries of 32 heads over 32 K tokens (8 kv
// heads, 1.07 TFLOP, causal) take 991 to 1044 us, 1.02 to 1.07 PFLOP/s; a bf16 product of 8192^3
// reaches 1.25.  The matrix unit is busy 55 % of the cycles, at 1.9 GHz of 2.4: the
// card's power holds the clock down, and codes are worked out and weights made
// meanwhile.  Few rows: 5 queries over 8 x 32 K tokens take 88 to 92 us, 3.2 to 3.3
// TB/s: a step is some 830 vector instructions of a wave, 640 of them to work out the
// values, 45 us of issue beside the 59 of a copy's rate; and a wave's codes, logits,
// weights and outputs are one chain, two waves a SIMD.  33 to 128 rows are between
// these: 9 to 16 queries over the same tokens take 195 us, one wave a SIMD, and
// waves without rows multiply as the others do.
//
// Rows are many or few.  Many: all waves of a workgroup share 64 tokens, worked
// out a step ahead into the other half of LDS.  At most 32 (k_chunk_few): each
// wave takes 64 tokens of its own, keys and values one after the other in LDS of
// its own, and they are joined at the end.  Where there are too few rows for the
// chip the tokens are shared among workgroups, by the steps that each row tile
// has, and k_chunk_join joins them.
#include <type_traits>

#include "quant4.h"

namespace mosaic {

namespace {

constexpr int CK_TILE = 64;                                // tokens of a step
constexpr int CK_SLOTS = 256;                              // workgroups that take part in splits, at most (one a compute unit)
constexpr int CK_ROWS = 256;                               // rows of a workgroup at most
constexpr int CK_FEW = 32, CK_FEW_WAVES = 8;
constexpr int CK_LEAST = 4;                                // steps of a share at least (of few rows: one for each wave)

// Weights are this power of two times as large.  fp16: those of 2^-25 and less of
// the row's largest would vanish, and a million of them count.  bf16: the running
// maximum is left behind by up to CK_LAG powers of two, as sums are multiplied
// through when it moves, and a weight past 1 times a value next to the type's
// largest would be infinite.
template <int DT> constexpr float CK_POW = DT ? -8.0f : 10.0f;
template <int DT> constexpr float CK_LAG = DT ? 8.0f : 4.0f;
static_assert(CK_POW<1> + CK_LAG<1> <= 0.0f, "bf16 weights are at most 1");

typedef __attribute__((ext_vector_type(16))) float cf16;
typedef __attribute__((ext_vector_type(2))) float cf2;
typedef __attribute__((ext_vector_type(2))) _Float16 ch2;
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

// s and both numbers of a pair
template <int DT> __device__ __forceinline__ float add2(uint32_t w, float s) {
    if constexpr (DT) {
        typedef __attribute__((ext_vector_type(2))) __bf16 b2;
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, w), __builtin_bit_cast(b2, 0x3f803f80u), s, false);
    } else {
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(ch2, w), __builtin_bit_cast(ch2, 0x3c003c00u), s, false);
    }
}

// Eight numbers in the order in which an operand holds them: as they are in
// bf16; 0, 4, 1, 5, 2, 6, 3, 7 in fp16, as two codes come out of one mask.
template <int DT> __device__ __forceinline__ uint4 dealt(uint4 w) {
    if constexpr (DT) return w;
    return make_uint4(__builtin_amdgcn_perm(w.z, w.x, 0x05040100u), __builtin_amdgcn_perm(w.z, w.x, 0x07060302u),
                      __builtin_amdgcn_perm(w.w, w.y, 0x05040100u), __builtin_amdgcn_perm(w.w, w.y, 0x07060302u));
}
template <int DT> __device__ __forceinline__ constexpr int deal(int i) { return DT ? i : (i >> 1) + 4 * (i & 1); }

// Grids of eight codes, ready for values(): fp32 numbers, or dealt fp16 pairs
template <int DT> struct Grid8;
template <> struct Grid8<1> {
    float s[8], z[8];
    __device__ __forceinline__ Grid8(uint4 sw, uint4 zw) {
        const uint32_t a[4] = {sw.x, sw.y, sw.z, sw.w}, b[4] = {zw.x, zw.y, zw.z, zw.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { s[i] = half_of<1>(a, i); z[i] = half_of<1>(b, i); }
    }
    // zero + scale * code, rounded (a code is, as an E4M3 byte, itself times 2^-9)
    __device__ __forceinline__ uint4 values(uint32_t c) const {
        const uint32_t lo = c & 0x0f0f0f0fu, hi = (c >> 4) & 0x0f0f0f0fu;
        const cf2 e0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, 512.0f, false), e1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, 512.0f, true);
        const cf2 o0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, 512.0f, false), o1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, 512.0f, true);
        return make_uint4(pack16<1>(fmaf(s[0], e0[0], z[0]), fmaf(s[1], o0[0], z[1])), pack16<1>(fmaf(s[2], e0[1], z[2]), fmaf(s[3], o0[1], z[3])),
                          pack16<1>(fmaf(s[4], e1[0], z[4]), fmaf(s[5], o1[0], z[5])), pack16<1>(fmaf(s[6], e1[1], z[6]), fmaf(s[7], o1[1], z[7])));
    }
};
template <> struct Grid8<0> {
    ch2 s[4], z[4];
    __device__ __forceinline__ Grid8(uint4 sw, uint4 zw) {
        sw = dealt<0>(sw);
        zw = dealt<0>(zw);
        __builtin_memcpy(s, &sw, 16);
        __builtin_memcpy(z, &zw, 16);
    }
    // the same in fp16, one rounding (a code's bits under 1024 are 1024 + code)
    __device__ __forceinline__ uint4 values(uint32_t c) const {
        const ch2 off = {(_Float16)1024.0f, (_Float16)1024.0f}, by = {(_Float16)0.0625f, (_Float16)0.0625f}, off16 = {(_Float16)-64.0f, (_Float16)-64.0f};
        uint32_t base = 0x64006400u;                       // (from a vector register: mask and base in one instruction)
        asm("" : "+v"(base));
        ch2 o[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t u = e ? c >> 8 : c;
            const ch2 a = __builtin_bit_cast(ch2, (u & 0x000f000fu) | base) - off;
            const ch2 b = __builtin_elementwise_fma(__builtin_bit_cast(ch2, (u & 0x00f000f0u) | base), by, off16);
            o[2 * e] = __builtin_elementwise_fma(s[2 * e], a, z[2 * e]);
            o[2 * e + 1] = __builtin_elementwise_fma(s[2 * e + 1], b, z[2 * e + 1]);
        }
        uint4 r;
        __builtin_memcpy(&r, o, 16);
        return r;
    }
};

// a row tile, and the workgroup's share of it
struct ChunkPlan {
    int p, s, h, row0;                                     // pair, its sequence and kv head, the tile's first row
    int L, m, nt;                                          // tokens, queries, steps of 64 (-1: no rows)
    int t0, t1;                                            // the share's steps
};
__device__ __forceinline__ ChunkPlan chunk_tile(const Q4Cache &q, const QChunk &c, int id, int tiles, int rows) {
    ChunkPlan r;
    const int pairs = q.S * q.H, t = tiles - 1 - id / pairs;       // (a pair's last tiles see most: first; one XCD's, if H is 8)
    r.p = id % pairs;
    r.s = r.p / q.H;
    r.h = r.p - r.s * q.H;
    r.row0 = t * rows;
    r.L = q.len(r.p);
    r.m = min(max(c.counts ? c.counts[r.s] : c.n, 0), c.n);
    const int last = min(r.m - 1, (r.row0 + rows - 1) / q.G);      // the tile's last query
    r.nt = r.row0 >= r.m * q.G ? -1 : (max(c.causal ? r.L - r.m + last + 1 : r.L, 0) + CK_TILE - 1) / CK_TILE;
    r.t0 = 0;
    r.t1 = r.nt;
    return r;
}

// Fewer tiles than CK_SLOTS: workgroups are dealt to them by their steps, as few
// for one as keep all shares of `per` steps (a multiple of STEP, at least LEAST)
// within CK_SLOTS.  Lengths are read on the device, so a captured launch follows
// them.  What workgroup w belongs to; one wave works it out, a lane holds up to
// four tiles in a row.
// (behind the shares' results: a tile's first workgroup, and how many it has)
__device__ __forceinline__ int2 *chunk_table(float *part) { return (int2 *)(part + (uint64_t)CK_SLOTS * CK_ROWS * (D + 4)); }
struct ChunkShare { int id, first, used, per; };           // tile (-1: none), its first workgroup, how many, steps of each
template <int STEP, int LEAST> __device__ __forceinline__ ChunkShare chunk_share(const Q4Cache &q, const QChunk &c, int tiles, int rows, int w) {
    const int units = q.S * q.H * tiles, lane = threadIdx.x & 63, K = (units + 63) / 64;
    int g[4] = {-1, -1, -1, -1};                           // steps in STEPs
    uint32_t sum = 0, most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int id = K * lane + j;
        if (j < K && id < units) {
            const int nt = chunk_tile(q, c, id, tiles, rows).nt;
            g[j] = nt < 0 ? -1 : (nt + STEP - 1) / STEP;
            sum += (uint32_t)min(max(g[j], 0), 1 << 23);
            most = max(most, (uint32_t)max(g[j], 0));
        }
    }
    sum = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(sum), 63);
    // g[j] / per rounded up, 1 at least (fp32's quotient is off by one at most)
    auto shares = [&](int j, uint32_t per) {
        const uint32_t y = (uint32_t)g[j] + per - 1u, k = (uint32_t)((float)y * __builtin_amdgcn_rcpf((float)per));
        const int rest = (int)(y - k * per);
        return g[j] < 0 ? 0u : max(1u, rest < 0 ? k - 1u : (rest >= (int)per ? k + 1u : k));
    };
    auto upto = [&](uint32_t per) {
        uint32_t n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < K) n += shares(j, per);
        return wave_scan_add(n);
    };
    auto fits = [&](uint32_t per) { return __builtin_amdgcn_readlane((int)upto(per), 63) <= CK_SLOTS; };
    uint32_t per = max((uint32_t)(LEAST / STEP), (sum + CK_SLOTS - 1) / CK_SLOTS);
    if (!fits(per)) {
        for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
        uint32_t no = per;
        per = (uint32_t)__builtin_amdgcn_readfirstlane((int)most);         // (one workgroup a tile)
        while (per - no > 1) {
            const uint32_t mid = (per + no) / 2;
            if (fits(mid)) per = mid; else no = mid;
        }
    }
    int first = (int)upto(per), id = -1, f = 0, used = 0;
#pragma unroll
    for (int j = 3; j >= 0; --j) {
        const int n = (int)shares(j, per);
        first -= n;
        if (w >= first && w < first + n) { id = K * lane + j; f = first; used = n; }
    }
    const uint64_t here = __ballot(id >= 0);
    if (here == 0) return ChunkShare{-1, 0, 0, 0};
    const int src = __builtin_ctzll(here);
    return ChunkShare{__builtin_amdgcn_readlane(id, src), __builtin_amdgcn_readlane(f, src), __builtin_amdgcn_readlane(used, src), (int)per * STEP};
}
__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }
// steps of each of a tile's ns shares
__device__ __forceinline__ int even_share(int nt, int ns, int step) { return max(div_up(div_up(nt, step), ns), 1) * step; }
// The workgroup's plan; used: how many workgroups its tile has (0: nothing to do).
// shared > 0: every tile has so many; < 0: they are dealt by the tiles' steps, and
// the first of a tile writes (first, used) to `table` for the join.
template <int STEP, int LEAST>
__device__ __forceinline__ ChunkPlan chunk_plan(const Q4Cache &q, const QChunk &c, int tiles, int rows, int shared, int2 *table, int &used) {
    __shared__ ChunkShare sh;
    if (shared < 0) {
        if (threadIdx.x < 64) {
            const ChunkShare x = chunk_share<STEP, LEAST>(q, c, tiles, rows, blockIdx.x);
            if (threadIdx.x == 0) {
                sh = x;
                if (x.id >= 0 && x.first == (int)blockIdx.x) table[x.id] = make_int2(x.first, x.used);
            }
        }
        __syncthreads();
    }
    const int ns = max(shared, 1), id = shared < 0 ? __builtin_amdgcn_readfirstlane(sh.id) : (int)blockIdx.x / ns;
    ChunkPlan r = chunk_tile(q, c, max(id, 0), tiles, rows);
    used = id < 0 || r.nt < 0 ? 0 : 1;
    if (shared && used) {
        const int per = shared < 0 ? __builtin_amdgcn_readfirstlane(sh.per) : even_share(r.nt, ns, STEP);
        r.t0 = ((int)blockIdx.x - (shared < 0 ? __builtin_amdgcn_readfirstlane(sh.first) : id * ns)) * per;
        r.t1 = min(r.nt, r.t0 + per);
        used = shared < 0 ? __builtin_amdgcn_readfirstlane(sh.used) : (r.t0 && r.t0 >= r.t1 ? 0 : div_up(max(r.nt, 1), per));
    }
    return r;
}

// A step's 64 keys (VALS: values) worked out by GT threads (thread gt) into LDS at
// `to`: keys by token, rows of 256 bytes, values by channel, rows of 128, with the
// 16-byte pieces of a row turned so that the operands' reads spread over the
// banks.  A thread takes eight codes a pass: channels 8 (gt % 16) + [0, 8) of a
// token, or tokens 8 (gt % 8) + [0, 8) of a channel.
template <int B, int DT, int GT, bool VALS> struct Step {
    static constexpr int R = VALS ? GT / 8 : GT / 16;      // channels or tokens of a pass
    static constexpr int P = (VALS ? D : CK_TILE) / R;     // passes
    static constexpr int NB = CK_TILE / B;                 // blocks of a step
    static constexpr int NG = VALS ? 1 : NB;               // grids of a thread
    static constexpr int GB = VALS ? 4 * B : 4 * D;        // bytes of a block's grids
    uint32_t c[P];
    uint4 g[NG][2];
    static __device__ __forceinline__ uint4 *at(uint8_t *to, int row, int piece) {
        return (uint4 *)(VALS ? to + row * 128 + 16 * (piece ^ ((row >> 1) & 7)) : to + row * 256 + 16 * (piece ^ (row & 15)));
    }
    // Codes and grids of step t; of one whose blocks are not whole, zeros.  (Through
    // buffer descriptors: a step is scalar work, and there is no branch, at whose end
    // the compiler would wait for what was loaded.  2048 queries over 32 K tokens
    // 1047 us with addresses in vector registers and the step's kind asked in the
    // loop, 1005 so.)
    __device__ __forceinline__ void load(const Q4Cache &q, uint64_t pb, int whole, int t, int gt) {
        const bool live = NB * (t + 1) <= whole;
        const uint64_t blk = pb + (live ? (uint32_t)(NB * t) : 0u);
        const auto codes = __builtin_amdgcn_make_buffer_rsrc((VALS ? q.v : q.k) + blk * (B * D / 2), 0, live ? CK_TILE * D / 2 : 0, 0x27000);
        const auto grids = __builtin_amdgcn_make_buffer_rsrc((uint8_t *)(VALS ? q.vg : q.kg) + blk * GB, 0, live ? NB * GB : 0, 0x27000);
        const int tok = 8 * (gt & 7), b = VALS ? tok / B : 0, ag = VALS ? b * GB + 2 * (tok % B) : 16 * (gt & 15);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            g[i][0] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(grids, ag + GB * i, 0, 0));
            g[i][1] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(grids, ag + GB * i + GB / 2, 0, 0));
        }
        const int ac = VALS ? b * (B * D / 2) + (gt >> 3) * (B / 2) + (tok % B) / 2 : 4 * gt;
#pragma unroll
        for (int i = 0; i < P; ++i) c[i] = __builtin_amdgcn_raw_buffer_load_b32(codes, ac + (VALS ? R * (B / 2) : 4 * GT) * i, 0, 0);
    }
    // a step of whole blocks
    __device__ __forceinline__ void store_full(int gt, uint8_t *to) const {
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            const Grid8<DT> gr(g[b][0], g[b][1]);
#pragma unroll
            for (int i = b * (P / NG); i < (b + 1) * (P / NG); ++i)
                *at(to, (VALS ? gt >> 3 : gt >> 4) + R * i, VALS ? gt & 7 : gt & 15) = gr.values(c[i]);
        }
    }
    // any step; the last one, with tokens of no whole block, is read here one pass
    // after the other, and tokens past the last are zeros
    __device__ __forceinline__ void store(const Q4Cache &q, int p, uint64_t pb, int whole, int tail, int t, int gt, uint8_t *to) const {
        if (NB * (t + 1) <= whole) {
            store_full(gt, to);
            return;
        }
        if constexpr (!VALS) {
            const int kc = gt & 15;
#pragma unroll 1
            for (int tk = gt >> 4; tk < CK_TILE; tk += R) {
                const int b = NB * t + tk / B;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (b < whole) {
                    const uint64_t blk = pb + (uint32_t)b;
                    const uint16_t *s = q.kg + blk * (2 * D) + 8 * kc;
                    x = Grid8<DT>(*(const uint4 *)s, *(const uint4 *)(s + D)).values(*(const uint32_t *)(q.k + blk * (B * D / 2) + (tk % B) * (D / 2) + 4 * kc));
                } else if (b == whole && tk % B < tail) {
                    x = dealt<DT>(*(const uint4 *)(q.kt + ((uint64_t)p * B + tk % B) * D + 8 * kc));
                }
                *at(to, tk, kc) = x;
            }
        } else {
            const int vo = gt & 7, b = NB * t + 8 * vo / B, pos = 8 * vo % B;
#pragma unroll 1
            for (int ch = gt >> 3; ch < D; ch += R) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (b < whole) {
                    const uint64_t blk = pb + (uint32_t)b;
                    const uint16_t *s = q.vg + blk * (2 * B) + pos;
                    x = Grid8<DT>(*(const uint4 *)s, *(const uint4 *)(s + B)).values(*(const uint32_t *)(q.v + blk * (B * D / 2) + ch * (B / 2) + pos / 2));
                } else if (b == whole) {
                    const int keep = tail - pos;           // tokens of the eight
                    if (keep > 0) x = *(const uint4 *)(q.vt + ((uint64_t)p * D + ch) * B + pos);
                    x.x = keep >= 2 ? x.x : (keep == 1 ? x.x & 0xffffu : 0u);
                    x.y = keep >= 4 ? x.y : (keep == 3 ? x.y & 0xffffu : 0u);
                    x.z = keep >= 6 ? x.z : (keep == 5 ? x.z & 0xffffu : 0u);
                    x.w = keep >= 8 ? x.w : (keep == 7 ? x.w & 0xffffu : 0u);
                    x = dealt<DT>(x);
                }
                *at(to, ch, vo) = x;
            }
        }
    }
};

// A wave's 32 rows: lanes l and l + 32 share row l % 32
template <int DT> struct Rows {
    uint4 qf[8];                                           // channels 16 e + 8 hl + [0, 8)
    cf16 acc[4];                                           // channel 32 ct + 8 (i / 4) + 4 hl + i % 4
    float m_run, l_run, mz, zs;                            // maximum, the lane's sum; what logits are lessened by, and scaled
    int seen;                                              // tokens that the row attends
    bool valid;
    __device__ __forceinline__ void begin(const Q4Cache &q, const QChunk &c, const ChunkPlan &pl, int row, int hl) {
        const int qi = row / q.G, head = pl.h * q.G + row - qi * q.G;
        valid = qi < pl.m;
        seen = valid ? (c.causal ? pl.L - pl.m + qi + 1 : pl.L) : 0;
        zs = powers_of(c.scale);
        const uint16_t *qp = c.q + pl.s * c.q_seq + qi * c.q_tok + head * c.q_head + 8 * hl;
        const uint32_t flip = flip_of(c.scale);
        const bool live = valid && c.scale != 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint4 w = live ? *(const uint4 *)(qp + 16 * e) : make_uint4(0, 0, 0, 0);
            qf[e] = dealt<DT>(make_uint4(w.x ^ flip, w.y ^ flip, w.z ^ flip, w.w ^ flip));
        }
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[ct][i] = 0.0f;
        m_run = -INFINITY;
        l_run = 0.0f;
        mz = CK_POW<DT>;
    }
    // What four matrix instructions take from LDS: of the values at vl, tokens 16 e
    // + 8 hl + [0, 8) of channels 32 ct + l32; of the keys at kl, channels 16 e + 8
    // hl + [0, 8), e = 2 g and 2 g + 1, of 32 tokens twice.  (Row r of the logits'
    // product is token (r & 16) + 8 (r / 4 & 1) + 4 (r / 8 & 1) + r % 4.)
    static __device__ __forceinline__ void read_v(const uint8_t *vl, int lane, int e, uint4 (&x)[4]) {
        const int l32 = lane & 31, hl = lane >> 5;
        const uint8_t *at = vl + l32 * 128 + ((16 * (hl ^ ((l32 >> 1) & 7))) ^ (32 * e));
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) x[ct] = *(const uint4 *)(at + 4096 * ct);
    }
    static __device__ __forceinline__ void read_k(const uint8_t *kl, int lane, int g, uint4 (&x)[4]) {
        const int l32 = lane & 31, hl = lane >> 5;
        const int tau = (l32 & 16) + 8 * ((l32 >> 2) & 1) + 4 * ((l32 >> 3) & 1) + (l32 & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *(const uint4 *)(kl + tau * 256 + ((16 * (hl ^ (tau & 15))) ^ (32 * (2 * g + (i >> 1)))) + 8192 * (i & 1));
    }
    __device__ __forceinline__ void mul_v(const uint4 (&x)[4], uint4 p) {
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) acc[ct] = mma32<DT>(x[ct], p, acc[ct]);
    }
    __device__ __forceinline__ void mul_k(const uint4 (&x)[4], int g, cf16 (&z)[2]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i & 1] = mma32<DT>(x[i], qf[2 * g + (i >> 1)], z[i & 1]);
    }
    // outputs of the weights pf over the values at `at` (V), or the logits z[n][i] of
    // token 32 n + 16 (i / 8) + 8 hl + i % 8 of the keys there; what an instruction
    // takes is read while the four before it run
    template <bool V> __device__ __forceinline__ void multiply(const uint8_t *at, const uint4 (&pf)[4], int lane, cf16 (&z)[2]) {
        uint4 x[2][4];
        if (V) read_v(at, lane, 0, x[0]); else read_k(at, lane, 0, x[0]);
        if (!V)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[n][i] = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (g < 3) { if (V) read_v(at, lane, g + 1, x[(g + 1) & 1]); else read_k(at, lane, g + 1, x[(g + 1) & 1]); }
            __builtin_amdgcn_sched_barrier(0);
            if (V) mul_v(x[g & 1], pf[g]); else mul_k(x[g & 1], g, z);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // the same, read as the compiler sees fit (fewer registers)
    __device__ __forceinline__ void multiply_v(const uint8_t *vl, const uint4 (&pf)[4], int lane) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint4 x[4];
            read_v(vl, lane, e, x);
            mul_v(x, pf[e]);
        }
    }
    __device__ __forceinline__ void multiply_k(const uint8_t *kl, int lane, cf16 (&z)[2]) const {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) z[n][i] = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint4 x[4];
            read_k(kl, lane, g, x);
            mul_k(x, g, z);
        }
    }
    // the softmax's step: weights of tokens 16 e + 8 hl + [0, 8), dealt
    __device__ __forceinline__ void weigh(cf16 (&z)[2], int t, int hl, bool masked, uint4 (&pf)[4]) {
        if (masked) {
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
        if (__any((cm - m_run) * zs > CK_LAG<DT>)) {
            const float mn = fmaxf(m_run, cm), mb = mn == -INFINITY ? 0.0f : mn;
            const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - mb) * zs);
            m_run = mn;
            mz = CK_POW<DT> - mb * zs;
            l_run *= alpha;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[ct][i] *= alpha;
        }
        // The sum is of the weights as they are rounded: a token that has nearly all
        // keeps its value.  A step's are summed before they meet the others': two
        // weights at a time would vanish next to one 2^25 times as large (a million of
        // them behind such a token: 1.6 % of the output).
        float ls = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(z[e >> 1][8 * (e & 1) + i], zs, mz));
            pf[e] = make_uint4(pack16<DT>(x[deal<DT>(0)], x[deal<DT>(1)]), pack16<DT>(x[deal<DT>(2)], x[deal<DT>(3)]),
                               pack16<DT>(x[deal<DT>(4)], x[deal<DT>(5)]), pack16<DT>(x[deal<DT>(6)], x[deal<DT>(7)]));
            ls = add2<DT>(pf[e].w, add2<DT>(pf[e].z, add2<DT>(pf[e].y, add2<DT>(pf[e].x, ls))));
        }
        l_run += ls;
    }
};

__device__ __forceinline__ uint16_t *out_row(const Q4Cache &q, const QChunk &c, const ChunkPlan &pl, int row) {
    const int qi = row / q.G, head = pl.h * q.G + row - qi * q.G;
    return c.out + pl.s * c.o_seq + qi * c.o_tok + head * c.o_head;
}
__device__ __forceinline__ float power_of(float m, float zs) { return m == -INFINITY ? m : m * zs; }

// grid (row tiles and pairs), or (shares of them) where `shared` is not 0; RW waves of 32 rows
template <int B, int DT, int RW>
__global__ void __launch_bounds__(64 * RW) __attribute__((amdgpu_waves_per_eu(2)))
k_chunk(Q4Cache q, QChunk c, int tiles, int shared, float *part) {
    constexpr int KB = CK_TILE * D * 2;                    // bytes of a step's keys, and of its values
    __shared__ __align__(16) uint8_t kl[2][KB], vl[2][KB];
    int used;
    const ChunkPlan pl = chunk_plan<1, CK_LEAST>(q, c, tiles, 32 * RW, shared, chunk_table(part), used);
    if (used == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = pl.t0, t1 = pl.t1;
    const int hl = lane >> 5, row = pl.row0 + 32 * wave + (lane & 31);
    const int all = c.causal ? pl.L - pl.m + pl.row0 / q.G + 1 : pl.L;     // tokens that every row of the workgroup attends
    const int whole = pl.L / B, tail = pl.L % B;
    const uint64_t pb = (uint64_t)pl.p * q.N;
    // Of eight waves the first four work out the keys, the others the values, before
    // the logits rather than after them, so that a SIMD's two waves differ.  Four
    // waves do both.  The first loop has no branch: its steps are whole, and every
    // row sees them.
    constexpr bool TWO = RW == 8;
    const int n = t1 - t0, gt = tid & 255;
    Rows<DT> r;
    r.begin(q, c, pl, row, hl);
    auto work = [&](auto values_first) {
        constexpr bool VALS = decltype(values_first)::value;
        Step<B, DT, 256, VALS> st;
        Step<B, DT, 256, true> sv;                         // (four waves' values)
        auto load = [&](int i) {
            const int t = t0 + min(i, n - 1);
            st.load(q, pb, whole, t, gt);
            if (!TWO) sv.load(q, pb, whole, t, gt);
        };
        auto store = [&](int i) {
            if (i >= n) return;
            st.store(q, pl.p, pb, whole, tail, t0 + i, gt, VALS ? vl[i & 1] : kl[i & 1]);
            if (!TWO) sv.store(q, pl.p, pb, whole, tail, t0 + i, gt, vl[i & 1]);
        };
        auto store_full = [&](int i) {
            st.store_full(gt, VALS ? vl[i & 1] : kl[i & 1]);
            if (!TWO) sv.store_full(gt, vl[i & 1]);
        };
        cf16 z[2];
        uint4 pf[4];
        load(0);
        store(0);
        load(1);
        int i = 0;
        const int plain = min(min(n - 1, whole * B / CK_TILE - t0 - 1), all / CK_TILE - t0);
        for (; i < plain; ++i) {
            lds_barrier();
            if (VALS) { store_full(i + 1); load(i + 2); }
            r.template multiply<false>(kl[i & 1], pf, lane, z);
            if (!VALS) { store_full(i + 1); load(i + 2); }
            r.weigh(z, t0 + i, hl, false, pf);
            r.template multiply<true>(vl[i & 1], pf, lane, z);
        }
        for (; i < n; ++i) {
            lds_barrier();
            if (VALS) { store(i + 1); load(i + 2); }
            r.template multiply<false>(kl[i & 1], pf, lane, z);
            if (!VALS) { store(i + 1); load(i + 2); }
            r.weigh(z, t0 + i, hl, CK_TILE * (t0 + i + 1) > all, pf);
            r.template multiply<true>(vl[i & 1], pf, lane, z);
        }
    };
    if (n > 0) {
        if (TWO && wave >= 4) work(std::true_type{});
        else work(std::false_type{});
    }
    const float l = halves(r.l_run, [](float a, float b) { return a + b; }), inv = share_of(l);
    if (used == 1) {
        if (!r.valid) return;
        uint16_t *op = out_row(q, c, pl, row) + 4 * hl;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(uint2 *)(op + 32 * ct + 8 * a) = make_uint2(pack16<DT>(r.acc[ct][4 * a] * inv, r.acc[ct][4 * a + 1] * inv),
                                                              pack16<DT>(r.acc[ct][4 * a + 2] * inv, r.acc[ct][4 * a + 3] * inv));
        return;
    }
    // a share's averages, and (maximum, sum)
    float *to = part + ((uint64_t)blockIdx.x * (32 * RW) + (row - pl.row0)) * (D + 4);
    if (hl == 0) *(float2 *)to = make_float2(power_of(r.m_run, r.zs), l);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *(float4 *)(to + 4 + 32 * ct + 8 * a + 4 * hl) = make_float4(r.acc[ct][4 * a] * inv, r.acc[ct][4 * a + 1] * inv,
                                                                         r.acc[ct][4 * a + 2] * inv, r.acc[ct][4 * a + 3] * inv);
}

// at most 32 rows: grid (pairs), or (shares of them)
template <int B, int DT>
__global__ void __launch_bounds__(64 * CK_FEW_WAVES) __attribute__((amdgpu_waves_per_eu(2)))
k_chunk_few(Q4Cache q, QChunk c, int shared, float *part) {
    constexpr int W = CK_FEW_WAVES, KB = CK_TILE * D * 2;
    __shared__ __align__(16) uint8_t lds[W][KB];
    __shared__ float ml[W][32][2];
    int used;
    const ChunkPlan pl = chunk_plan<W, W>(q, c, 1, CK_FEW, shared, chunk_table(part), used);
    if (used == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = pl.t0, t1 = pl.t1;
    const int l32 = lane & 31, hl = lane >> 5;
    const int all = c.causal ? pl.L - pl.m + 1 : pl.L;     // tokens that every row attends
    const int whole = pl.L / B, tail = pl.L % B;
    const uint64_t pb = (uint64_t)pl.p * q.N;
    uint8_t *mine = lds[wave];
    Step<B, DT, 64, false> sk;
    Step<B, DT, 64, true> sv;
    int t = t0 + wave;
    sk.load(q, pb, whole, t, lane);
    sv.load(q, pb, whole, t, lane);
    Rows<DT> r;
    r.begin(q, c, pl, l32, hl);
    auto step = [&](auto any) {                            // any: also one whose blocks are not whole
        constexpr bool ANY = decltype(any)::value;
        cf16 z[2];
        uint4 pf[4];
        if (ANY) sk.store(q, pl.p, pb, whole, tail, t, lane, mine); else sk.store_full(lane, mine);
        mem_fence_compiler();
        wave_sync();
        if (!ANY) sk.load(q, pb, whole, t + W < t1 ? t + W : t, lane);
        r.multiply_k(mine, lane, z);
        mem_fence_compiler();
        wave_sync();
        if (ANY) sv.store(q, pl.p, pb, whole, tail, t, lane, mine); else sv.store_full(lane, mine);
        mem_fence_compiler();
        wave_sync();                                       // (the wave's LDS operations run in their order)
        if (!ANY) sv.load(q, pb, whole, t + W < t1 ? t + W : t, lane);
        r.weigh(z, t, hl, CK_TILE * (t + 1) > all, pf);
        r.multiply_v(mine, pf, lane);
        mem_fence_compiler();
        wave_sync();
    };
    const int full = min(t1, whole * B / CK_TILE);
    for (; t < full; t += W) step(std::false_type{});
    if (t < t1) step(std::true_type{});                    // (the last step of all)
    // the waves joined, in their order; each takes 16 channels
    float l = halves(r.l_run, [](float a, float b) { return a + b; });
    float *sums = (float *)mine;                           // [channel][row]
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(32 * ct + 8 * (i >> 2) + 4 * hl + (i & 3)) * 32 + l32] = r.acc[ct][i];
    if (hl == 0) { ml[wave][l32][0] = r.m_run; ml[wave][l32][1] = l; }
    __syncthreads();
    float m = -INFINITY, f[W], x[8];
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, ml[w][l32][0]);
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        f[w] = ml[w][l32][0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ml[w][l32][0] - m) * r.zs);
        l += f[w] * ml[w][l32][1];
    }
    const float inv = share_of(l);
#pragma unroll
    for (int i = 0; i < 8; ++i) {                          // channels 16 wave + 8 hl + i
        x[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) x[i] += f[w] * ((const float *)lds[w])[(16 * wave + 8 * hl + i) * 32 + l32];
        x[i] *= inv;
    }
    if (used == 1) {
        if (r.valid)
            *(uint4 *)(out_row(q, c, pl, l32) + 16 * wave + 8 * hl) = make_uint4(pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]), pack16<DT>(x[4], x[5]),
                                                                                 pack16<DT>(x[6], x[7]));
        return;
    }
    float *to = part + ((uint64_t)blockIdx.x * CK_FEW + l32) * (D + 4);
    if (wave == 0 && hl == 0) *(float2 *)to = make_float2(power_of(m, r.zs), l);
    *(float4 *)(to + 4 + 16 * wave + 8 * hl) = make_float4(x[0], x[1], x[2], x[3]);
    *(float4 *)(to + 8 + 16 * wave + 8 * hl) = make_float4(x[4], x[5], x[6], x[7]);
}

// the shares of a row tile joined, in their order; grid (row tiles and pairs, rows / 8), 32 lanes a row
template <int DT>
__global__ void __launch_bounds__(256) k_chunk_join(Q4Cache q, QChunk c, int tiles, int rows, int shared, float *part) {
    const ChunkPlan pl = chunk_tile(q, c, blockIdx.x, tiles, rows);
    // (a tile without rows has no entry, and writes nothing)
    const int2 sh = shared < 0 ? chunk_table(part)[blockIdx.x]
                               : make_int2((int)blockIdx.x * shared, div_up(max(pl.nt, 1), even_share(pl.nt, shared, rows == CK_FEW ? CK_FEW_WAVES : 1)));
    if (sh.y <= 1) return;
    const int r = 8 * blockIdx.y + (threadIdx.x >> 5), ch = 4 * (threadIdx.x & 31);
    const int row = pl.row0 + r, qi = row / q.G, head = pl.h * q.G + row - qi * q.G;
    if (qi >= pl.m) return;
    const float *from = part + (uint64_t)sh.x * rows * (D + 4) + r * (D + 4);
    float M = -INFINITY, S = 0.0f;
    float4 A = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < sh.y; ++k) {
        const float *o = from + (uint64_t)k * rows * (D + 4);
        const float2 x = *(const float2 *)o;
        const float4 a = *(const float4 *)(o + 4 + ch);
        const float mn = fmaxf(M, x.x), mb = mn == -INFINITY ? 0.0f : mn;
        float f = S * __builtin_amdgcn_exp2f(M - mb), g = x.y * __builtin_amdgcn_exp2f(x.x - mb);
        S = f + g;
        const float inv = share_of(S);
        f *= inv;
        g *= inv;
        A = make_float4(A.x * f + a.x * g, A.y * f + a.y * g, A.z * f + a.z * g, A.w * f + a.w * g);
        M = mn;
    }
    *(uint2 *)(c.out + pl.s * c.o_seq + qi * c.o_tok + head * c.o_head + ch) = make_uint2(pack16<DT>(A.x, A.y), pack16<DT>(A.z, A.w));
}

}  // namespace

size_t quant4_chunk_ws_bytes(int pairs, int blocks, int block) {
    // (nothing where no launch shares its tiles: as many pairs as slots, or tokens for one share)
    if (pairs >= CK_SLOTS || ceil_div(blocks, CK_TILE / block) <= CK_LEAST) return 0;
    return (size_t)CK_SLOTS * (CK_ROWS * (D + 4) * sizeof(float) + sizeof(int2));
}

hipError_t launch_quant4_chunk(const Q4Cache &q, int block, int dtype, const QChunk &c, float *part, hipStream_t s) {
    const int pairs = q.S * q.H, all = c.n * q.G;
    const int rows = all <= CK_FEW ? CK_FEW : (all <= 128 ? 128 : CK_ROWS), tiles = (all + rows - 1) / rows;
    const long long wgs = (long long)pairs * tiles;
    // us of 6 x 1500 tokens, 448 rows, 72 pairs: 128 rows a workgroup 60.2, 256 49.8; 1 x 8 K, 256 rows, 8 pairs, best
    // splits: 128 34.2, 256 36.6; 4 x 4 K, 400 rows, 32 pairs: 128 55.4, 256 50.7.  32 rows alone go to k_chunk_few.
    // More workgroups than compute units run one after the other, and their parts are memory traffic (6 x 1500 tokens,
    // 144 tiles, 49.8 with one workgroup each, 73.6 with two), so tiles are shared among as many as there are units.
    // A sequence alone: evenly (1 x 2 K, 2048 rows, 64 tiles, 58.2 / 36.7 / 52.5 with one, four and eight a tile).  Several:
    // by their steps, as they may differ.  Evenly / by steps, ragged batches: 6 x up to 1500 tokens 50.2 / 45.2, 5 queries
    // over 8 x up to 32 K 74 / 56, over 16 x up to 8 K 43.0 / 38.2; batches of one length pay for the dealing, 5 over 8 x 32 K
    // 84.5 / 84, 100 over 4 x 4 K 49.7 / 50.4, 5 over 24 x 8 K (192 tiles, not shared, not joined) 69.5 / 73.3, 6 x 1500 51 / 57.
    const int least = rows == CK_FEW ? CK_FEW_WAVES : CK_LEAST, most = ceil_div(ceil_div(q.N, CK_TILE / block), least);
    const int ns = wgs < CK_SLOTS ? (most < CK_SLOTS / (int)wgs ? most : CK_SLOTS / (int)wgs) : 1;
    const int shared = wgs >= CK_SLOTS || most == 1 || (q.S == 1 && ns == 1) ? 0 : (q.S == 1 ? ns : -1);
    const long long all_shares = shared < 0 ? wgs * most : wgs * ns;
    const dim3 grid((uint32_t)(shared < 0 && all_shares > CK_SLOTS ? CK_SLOTS : all_shares));
    auto by_rows = [&](auto b, auto dt) {
        constexpr int BL = decltype(b)::value, T = decltype(dt)::value;
        if (rows == CK_FEW) hipLaunchKernelGGL((k_chunk_few<BL, T>), grid, dim3(64 * CK_FEW_WAVES), 0, s, q, c, shared, part);
        else if (rows == 128) hipLaunchKernelGGL((k_chunk<BL, T, 4>), grid, dim3(256), 0, s, q, c, tiles, shared, part);
        else hipLaunchKernelGGL((k_chunk<BL, T, 8>), grid, dim3(512), 0, s, q, c, tiles, shared, part);
    };
    auto by_type = [&](auto b) { if (dtype) by_rows(b, std::integral_constant<int, 1>{}); else by_rows(b, std::integral_constant<int, 0>{}); };
    if (block == 32) by_type(std::integral_constant<int, 32>{}); else by_type(std::integral_constant<int, 64>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !shared) return e;
    const dim3 jgrid((uint32_t)wgs, rows / 8);
    if (dtype) hipLaunchKernelGGL(k_chunk_join<1>, jgrid, dim3(256), 0, s, q, c, tiles, rows, shared, part);
    else hipLaunchKernelGGL(k_chunk_join<0>, jgrid, dim3(256), 0, s, q, c, tiles, rows, shared, part);
    return hipGetLastError();
}

}  // namespace mosaic
