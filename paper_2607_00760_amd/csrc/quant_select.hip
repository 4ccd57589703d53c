// quant_select.hip -- which blocks of the 8-bit cache a query attends
// (mosaic_quant_select_attention).
//
// A block's bounds give the largest product that any of its keys can have with
// a query: sum over channels of q_c hi_c where q_c > 0 and q_c lo_c elsewhere.
// With q in 8-bit integers that is an integer product of [max(q, 0), min(q, 0)]
// with [hi, lo], 256 long: one 16x16x64 integer matrix product for each quarter
// gives 16 blocks x 16 heads, exact in any order, so the selection does not
// depend on how the work is split.  The score is that integer times the
// query's scale, the largest over the group's heads, times the bounds' unit.
// 260 bytes of a block are read, a thirtieth of its codes.
#include "topk.h"
#include "quant.h"

namespace mosaic {

namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int QS_UNIT = 64;                                // blocks of a scoring workgroup's step, 16 a wave
constexpr int QS_RUNS = 1024;                              // runs of a scoring launch, about

// codes of 16 channels of a query in 8-bit integers, one half of them zeroed
__device__ __forceinline__ i32x4 pack_signed(const float (&x)[16], bool upper) {
    i32x4 r;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t u = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (int)x[4 * w + i];
            u |= ((uint32_t)(upper ? max(c, 0) : min(c, 0)) & 0xffu) << (8 * i);
        }
        r[w] = (int)u;
    }
    return r;
}

// The scores of blocks [b, b1) of pair p (nb blocks), a wave's 16 from b and
// then every `step`: emit(block, score).  AHEAD steps are in flight, the
// first before the query is looked at.  (Loads past the end read the last
// block again: a branch around each would wait for those before it.)
template <int DT, int AHEAD, typename E>
__device__ __forceinline__ void score_blocks(const QCache &q, int p, int nb, const uint16_t *query, int b, int b1, int step, E emit) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, q4 = lane >> 4;
    const int8_t *bp = q.bounds + (uint64_t)p * q.N * (2 * D);
    const float *bs = q.bs + (uint64_t)p * q.N;
    if (b >= b1) return;
    i32x4 w[AHEAD][4];
    float u[AHEAD];                                     // of block 4 q4 + l16 % 4
    auto load = [&](int s, int at) {
        const i32x4 *row = (const i32x4 *)(bp + (uint64_t)min(at + l16, nb - 1) * (2 * D)) + q4;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[s][e] = row[4 * e];
        u[s] = bs[min(at + 4 * q4 + (l16 & 3), nb - 1)];
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) load(s, b + s * step);
    const int head = min(l16, q.G - 1);                    // columns past the group repeat its last head
    const uint16_t *qp = query + ((uint64_t)p * q.G + head) * D;
    float x[2][16];
    float a = 0.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        uint16_t h[16];
        __builtin_memcpy(h, __builtin_assume_aligned(qp + 64 * e + 16 * q4, 16), 32);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[e][i] = h2f(h[i], DT);
            a = fmaxf(a, fabsf(x[e][i]));
        }
    }
    a = fmaxf(rows_all(a, [](float m, float o) { return fmaxf(m, o); }), QLEAST);
    const float inv = 127.0f / a, unit = a / 127.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[e][i] = rintf(x[e][i] * inv);
    const i32x4 qb[4] = {pack_signed(x[0], true), pack_signed(x[1], true), pack_signed(x[0], false), pack_signed(x[1], false)};
    auto score = [&](int s, int at) {
        i32x4 acc = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s][e], qb[e], acc, 0, 0, 0);
        float sc[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {                      // block at + 4 q4 + r: the largest over the heads
            sc[r] = (float)acc[r] * unit;
            sc[r] = fmaxf(sc[r], dpp_read<0x128, 0xf>(sc[r]));
            sc[r] = fmaxf(sc[r], dpp_read<0x124, 0xf>(sc[r]));
            sc[r] = fmaxf(sc[r], dpp_read<0x122, 0xf>(sc[r]));
            sc[r] = fmaxf(sc[r], dpp_read<0x121, 0xf>(sc[r]));
        }
        const float mine = (l16 & 2) ? ((l16 & 1) ? sc[3] : sc[2]) : ((l16 & 1) ? sc[1] : sc[0]);
        const int blk = at + 4 * q4 + l16;
        if (l16 < 4 && blk < b1) emit(blk, mine * u[s]);
    };
    for (; b + AHEAD * step < b1; b += AHEAD * step)
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            score(s, b + s * step);
            load(s, b + (s + AHEAD) * step);
        }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) score(s, b + s * step);
}

// grid QS_RUNS + pairs: one run of 64-block units of a pair each
template <int DT>
__global__ void __launch_bounds__(256) k_quant_score(QCache q, int block, const uint16_t *query, float *scores, int32_t *list) {
    const QPlan pl = q_plan(q, QShare{QS_RUNS, QS_RUNS, 1, 2, 1, 0, 0, 0}, [&](int L) { return (L / block + QS_UNIT - 1) / QS_UNIT; }, blockIdx.x);
    if (!pl.live) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int p = pl.s * q.H + pl.h, nb = pl.L / block;
    const int b0 = pl.i * pl.c * QS_UNIT, b1 = min(nb, b0 + pl.c * QS_UNIT);
    {                                                      // the list's places, -1 until the selection takes them
        int32_t *lp = list + (uint64_t)p * q.N;
        const int e1 = pl.i == pl.ns - 1 ? q.N : b1;
        for (int e = b0 + threadIdx.x; e < e1; e += 256) lp[e] = -1;
    }
    float *out = scores + (uint64_t)p * q_score_stride(q.N);
    auto emit = [&](int at, float s) { out[at] = s; };
    if (pl.c == 1) score_blocks<DT, 1>(q, p, nb, query, b0 + 16 * wave, b1, QS_UNIT, emit);
    else score_blocks<DT, 2>(q, p, nb, query, b0 + 16 * wave, b1, QS_UNIT, emit);
}

// The `want` (at least one) best of a pair's scores src[0, nb), by one workgroup
// of NW waves: thread t owns the KPT consecutive blocks from KPT t (KPT = 0: as
// many as it takes, read again in each pass).  A radix selection over the range
// of the keys: a pass of 2048 bins narrows the candidates to the threshold's
// bin; where that holds up to 64 of them (mostly after the first) the waves
// rank them, a lane each.  Blocks above the threshold are taken, those equal to
// it in block order while they are needed; one scan places them in ascending
// order.
constexpr int QK_BINS = 2048, QK_FEW = 64;
template <int QK_NW> struct PickSmem {
    uint32_t hist[2][QK_BINS];
    uint32_t mm[2 * QK_NW], pk[QK_NW], pub[3], sc[2][QK_NW], few[QK_FEW], cmp[QK_FEW], nfew;
};
template <int KPT, int NW>
__device__ __forceinline__ void pick(const float *src, int nb, int want, int32_t *dst, PickSmem<NW> &sm) {
    constexpr int NT = 64 * NW, BINS = QK_BINS, BPT = BINS / NT, FEW = QK_FEW;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int own = KPT ? KPT : (nb + NT - 1) / NT;
    const int i0 = min(nb, tid * own), n_own = min(nb, i0 + own) - i0;
    uint32_t kr[KPT ? KPT : 1];
    if (KPT) {
        float4 f[KPT ? KPT / 4 : 1];
#pragma unroll
        for (int e = 0; e < KPT / 4; ++e) f[e] = 4 * e < n_own ? *(const float4 *)(src + i0 + 4 * e) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int e = 0; e < KPT / 4; ++e) {
            kr[4 * e] = score_key(f[e].x);
            kr[4 * e + 1] = score_key(f[e].y);
            kr[4 * e + 2] = score_key(f[e].z);
            kr[4 * e + 3] = score_key(f[e].w);
        }
    }
    for (int i = tid; i < BINS; i += NT) sm.hist[0][i] = 0u;
    if (tid == 0) sm.nfew = 0u;
    if (tid < FEW) sm.cmp[tid] = 0u;
    auto each = [&](auto f) {
        if (KPT) {
#pragma unroll
            for (int e = 0; e < (KPT ? KPT : 1); ++e)
                if (e < n_own) f(e, kr[e]);
        } else {
            for (int e = 0; e < n_own; ++e) f(e, score_key(src[i0 + e]));
        }
    };
    uint32_t kmin = 0xffffffffu, kmax = 0u;
    each([&](int, uint32_t k) { kmin = min(kmin, k); kmax = max(kmax, k); });
    kmin = ~wave_max_u(~kmin);
    kmax = wave_max_u(kmax);
    if (lane == 0) { sm.mm[wv] = kmin; sm.mm[NW + wv] = kmax; }
    lds_barrier();
    kmin = ~wave_max_u(lane < NW ? ~sm.mm[lane] : 0u);
    kmax = wave_max_u(lane < NW ? sm.mm[NW + lane] : 0u);
    uint32_t base = kmin, span = kmax - kmin, rem = (uint32_t)want;    // candidates: [base, base + span]
    for (int pass = 0;; ++pass) {
        uint32_t *hc = sm.hist[pass & 1], *hn = sm.hist[(pass + 1) & 1];
        const int bits = 32 - (span ? __builtin_clz(span) : 32), sh = bits > 11 ? bits - 11 : 0;
        each([&](int, uint32_t k) { if (k >= base && k - base <= span) atomicAdd(&hc[(k - base) >> sh], 1u); });
        lds_barrier();
        uint32_t hb[BPT], mine = 0u;                       // the thread's bins, from the top down
        const int b0 = BINS - BPT * (tid + 1);
#pragma unroll
        for (int e = 0; e < BPT; ++e) { hb[e] = hc[b0 + e]; mine += hb[e]; hn[b0 + e] = 0u; }
        uint32_t tot;
        uint32_t above = block_excl<NW>(mine, tot, sm.pk);
        if (above < rem && above + mine >= rem) {
#pragma unroll
            for (int e = BPT - 1; e >= 0; --e) {
                if (above < rem && above + hb[e] >= rem) { sm.pub[0] = (uint32_t)(b0 + e); sm.pub[1] = rem - above; sm.pub[2] = hb[e]; }
                above += hb[e];
            }
        }
        lds_barrier();
        base += sm.pub[0] << sh;
        span = min(span - (sm.pub[0] << sh), sh ? (1u << sh) - 1u : 0u);
        rem = sm.pub[1];
        if (sh == 0) break;                                // single keys: the threshold is base
        if (sm.pub[2] <= FEW) {                            // (once: the loop ends here)
            const int n = (int)sm.pub[2];
            each([&](int, uint32_t k) { if (k >= base && k - base <= span) sm.few[atomicAdd(&sm.nfew, 1u)] = k; });
            lds_barrier();
            // a wave compares every candidate, a lane each, with its share of them
            const uint32_t k = lane < n ? sm.few[lane] : 0u;
            uint32_t c = 0u;                               // candidates above, and from bit 16 equal ones
            for (int e = wv; e < n; e += NW) {
                const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)k, e);
                c += o > k ? 1u : (o == k ? 0x10000u : 0u);
            }
            if (c) atomicAdd(&sm.cmp[lane], c);
            lds_barrier();
            const uint32_t gt = sm.cmp[lane] & 0xffffu, ge = gt + (sm.cmp[lane] >> 16);
            const int l = (int)__builtin_ctzll(__ballot(lane < n && gt < rem && ge >= rem));   // (rem of the n are needed: never empty)
            base = (uint32_t)__builtin_amdgcn_readlane((int)k, l);
            rem -= (uint32_t)__builtin_amdgcn_readlane((int)gt, l);
            break;
        }
    }
    // taken: above the threshold, or equal to it while the equal ones before are fewer than rem
    uint32_t eq = 0u, gt = 0u, tot;
    each([&](int, uint32_t k) { eq += k == base ? 1u : 0u; gt += k > base ? 1u : 0u; });
    uint32_t before = block_excl<NW>(eq, tot, sm.sc[0]);
    uint32_t pos = block_excl<NW>(gt + min(eq, rem > before ? rem - before : 0u), tot, sm.sc[1]);
    each([&](int e, uint32_t k) {
        const bool t = k > base || (k == base && before < rem);
        before += k == base ? 1u : 0u;
        if (t) dst[pos++] = i0 + e;
    });
}

template <int KPT>
__global__ void __launch_bounds__(1024) k_quant_topk(QCache q, int block, int num, int den, const float *scores, int32_t *list) {
    __shared__ PickSmem<16> sm;
    const int p = blockIdx.x, nb = q.len(p) / block, want = q_want(nb, num, den);
    int32_t *dst = list + (uint64_t)p * q.N;
    if (want == 0) {                                       // (no scores were made)
        for (int i = threadIdx.x; i < q.N; i += 1024) dst[i] = -1;
        return;
    }
    pick<KPT, 16>(scores + (uint64_t)p * q_score_stride(q.N), nb, want, dst, sm);
}

// Scores and selection of a pair of up to QK_FUSED blocks in one workgroup, the
// scores in LDS.  It saves a launch (2 us), and a compute unit reads 32 bytes a
// ns at most, whoever asks: so for caches of up to 256 blocks a pair, and for
// larger ones where there are pairs for half of the chip.  Whole calls, blocks
// of 32, 8 kv heads, us in one workgroup / spread over several:
//   tokens         2048         8192         16384        32768
//   1 sequence     13.0 / 14.6  16.2 / 17.5  18.0 / 17.4  22.3 / 18.2
//   32             13.8 / 15.4  20.7 / 23.5  35.3 / 37.6  59.9 / 63.3
constexpr int QK_FUSED = 1024, QK_NW = 4;
template <int DT>
__global__ void __launch_bounds__(64 * QK_NW) k_quant_pick(QCache q, int block, const uint16_t *query, int num, int den, int32_t *list) {
    __shared__ PickSmem<QK_NW> sm;
    __shared__ __align__(16) float scores[QK_FUSED];
    const int p = blockIdx.x, nb = q.len(p) / block, want = q_want(nb, num, den);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t *dst = list + (uint64_t)p * q.N;
    for (int i = want + threadIdx.x; i < q.N; i += 64 * QK_NW) dst[i] = -1;
    if (want == 0) return;
    score_blocks<DT, 4>(q, p, nb, query, 16 * wave, nb, 16 * QK_NW, [&](int at, float s) { scores[at] = s; });
    lds_barrier();
    pick<4, QK_NW>(scores, nb, want, dst, sm);
}

}  // namespace

hipError_t launch_quant_select(const QCache &q, int block, int dtype, const uint16_t *query, int num, int den, float *scores,
                               int32_t *list, hipStream_t s) {
    const int pairs = q.S * q.H;
    if (q.N <= 256 || (q.N <= QK_FUSED && pairs >= 128)) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pairs), dim3(64 * QK_NW), 0, s, q, block, query, num, den, list); };
        if (dtype) go(k_quant_pick<1>); else go(k_quant_pick<0>);
        return hipGetLastError();
    }
    const long long most = (long long)pairs * ceil_div(q.N, QS_UNIT);
    const dim3 grid((uint32_t)(most < QS_RUNS + pairs ? most : QS_RUNS + pairs));
    if (dtype) hipLaunchKernelGGL(k_quant_score<1>, grid, dim3(256), 0, s, q, block, query, scores, list);
    else hipLaunchKernelGGL(k_quant_score<0>, grid, dim3(256), 0, s, q, block, query, scores, list);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pairs), dim3(1024), 0, s, q, block, num, den, scores, list); };
    if (q.N <= 4 * 1024) go(k_quant_topk<4>);
    else if (q.N <= 16 * 1024) go(k_quant_topk<16>);
    else if (q.N <= 32 * 1024) go(k_quant_topk<32>);
    else go(k_quant_topk<0>);
    return hipGetLastError();
}

}  // namespace mosaic
