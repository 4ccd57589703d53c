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

constexpr int QS_UNIT = 64;                                // blocks of a workgroup's step, 16 a wave
constexpr int QS_RUNS = 1024;                              // runs of a launch, about
constexpr int QS_AHEAD = 4;

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

// grid QS_RUNS + pairs: one run of 64-block units of a pair each.  A wave has
// QS_AHEAD steps of 16 blocks in flight; the first are out before the query is
// looked at.
template <int DT>
__global__ void __launch_bounds__(256) k_quant_score(QCache q, int block, const uint16_t *query, float *scores, int32_t *list) {
    const QPlan pl = q_plan(q, QS_RUNS, 1, 1, 0, [&](int L) { return (L / block + QS_UNIT - 1) / QS_UNIT; }, blockIdx.x);
    if (!pl.live) return;
    const int lane = threadIdx.x & 63, l16 = lane & 15, q4 = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int p = pl.s * q.H + pl.h, nb = pl.L / block;
    const int8_t *bp = q.bounds + (uint64_t)p * q.N * (2 * D);
    const float *bs = q.bs + (uint64_t)p * q.N;
    float *out = scores + (uint64_t)p * q_score_stride(q.N);
    int b = pl.i * pl.c * QS_UNIT + 16 * wave;
    const int b1 = min(nb, (pl.i + 1) * pl.c * QS_UNIT);
    i32x4 w[QS_AHEAD][4];
    float u[QS_AHEAD][4];
    auto load = [&] {
#pragma unroll
        for (int a = 0; a < QS_AHEAD; ++a) {
            const int at = b + a * QS_UNIT;
            if (at < b1) {
                const i32x4 *row = (const i32x4 *)(bp + (uint64_t)min(at + l16, nb - 1) * (2 * D)) + q4;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[a][e] = row[4 * e];
#pragma unroll
                for (int r = 0; r < 4; ++r) u[a][r] = bs[min(at + 4 * q4 + r, nb - 1)];
            }
        }
    };
    load();
    {                                                      // the list's places, -1 until the selection takes them
        int32_t *lp = list + (uint64_t)p * q.N;
        const int e1 = pl.i == pl.ns - 1 ? q.N : b1;
        for (int e = pl.i * pl.c * QS_UNIT + threadIdx.x; e < e1; e += 256) lp[e] = -1;
    }
    const int head = min(l16, q.G - 1);                    // columns past the group repeat its last head
    const uint16_t *qp = query + ((uint64_t)p * q.G + head) * D;
    float x[2][16];
    float a = 0.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[e][i] = h2f(qp[64 * e + 16 * q4 + i], DT);
            a = fmaxf(a, fabsf(x[e][i]));
        }
    a = fmaxf(rows_all(a, [](float m, float o) { return fmaxf(m, o); }), QLEAST);
    const float inv = 127.0f / a, unit = a / 127.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[e][i] = rintf(x[e][i] * inv);
    const i32x4 qb[4] = {pack_signed(x[0], true), pack_signed(x[1], true), pack_signed(x[0], false), pack_signed(x[1], false)};
    while (b < b1) {
#pragma unroll
        for (int s = 0; s < QS_AHEAD; ++s) {
            if (b + s * QS_UNIT >= b1) break;
            i32x4 acc = i32x4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s][e], qb[e], acc, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {                  // block at + 4 q4 + r, head l16
                float sc = (float)acc[r] * unit;
                sc = fmaxf(sc, dpp_read<0x128, 0xf>(sc));
                sc = fmaxf(sc, dpp_read<0x124, 0xf>(sc));
                sc = fmaxf(sc, dpp_read<0x122, 0xf>(sc));
                sc = fmaxf(sc, dpp_read<0x121, 0xf>(sc));
                const int at = b + s * QS_UNIT + 4 * q4 + r;
                if (l16 == r && at < b1) out[at] = sc * u[s][r];
            }
        }
        b += QS_AHEAD * QS_UNIT;
        if (b < b1) load();
    }
}

// The `want` best scores of a pair, one workgroup of 16 waves: thread t owns
// the KPT consecutive blocks from KPT t (KPT = 0: as many as it takes, read
// again from memory in each pass).  A radix selection over the range of the
// keys: a pass of 2048 bins narrows the candidates to the threshold's bin;
// where that holds up to 64 of them (mostly after the first) every wave ranks
// them itself, a lane each.  Blocks above the threshold are taken, those equal
// to it in block order while they are needed; one scan places them in
// ascending order.
template <int KPT>
__global__ void __launch_bounds__(1024) k_quant_topk(QCache q, int block, int num, int den, const float *scores, int32_t *list) {
    constexpr int NW = 16, NT = 64 * NW, BINS = 2048, BPT = BINS / NT, FEW = 64;
    __shared__ uint32_t hist[2][BINS];
    __shared__ uint32_t mm[2 * NW], pk[NW], pub[3], sc[2][NW], few[FEW], cmp[FEW], nfew;
    const int p = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int nb = q.len(p) / block, want = q_want(nb, num, den);
    const float *src = scores + (uint64_t)p * q_score_stride(q.N);
    int32_t *dst = list + (uint64_t)p * q.N;
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
    for (int i = tid; i < BINS; i += NT) hist[0][i] = 0u;
    if (tid == 0) nfew = 0u;
    if (tid < FEW) cmp[tid] = 0u;
    if (want == 0) {                                       // (no scores were made)
        for (int i = tid; i < q.N; i += NT) dst[i] = -1;
        return;
    }
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
    if (lane == 0) { mm[wv] = kmin; mm[NW + wv] = kmax; }
    lds_barrier();
    kmin = ~wave_max_u(lane < NW ? ~mm[lane] : 0u);
    kmax = wave_max_u(lane < NW ? mm[NW + lane] : 0u);
    uint32_t base = kmin, span = kmax - kmin, rem = (uint32_t)want;    // candidates: [base, base + span]
    for (int pass = 0;; ++pass) {
        uint32_t *hc = hist[pass & 1], *hn = hist[(pass + 1) & 1];
        const int bits = 32 - (span ? __builtin_clz(span) : 32), sh = bits > 11 ? bits - 11 : 0;
        each([&](int, uint32_t k) { if (k >= base && k - base <= span) atomicAdd(&hc[(k - base) >> sh], 1u); });
        lds_barrier();
        uint32_t hb[BPT], mine = 0u;                       // the thread's bins, from the top down
        const int b0 = BINS - BPT * (tid + 1);
#pragma unroll
        for (int e = 0; e < BPT; ++e) { hb[e] = hc[b0 + e]; mine += hb[e]; hn[b0 + e] = 0u; }
        uint32_t tot;
        uint32_t above = block_excl<NW>(mine, tot, pk);
        if (above < rem && above + mine >= rem) {
#pragma unroll
            for (int e = BPT - 1; e >= 0; --e) {
                if (above < rem && above + hb[e] >= rem) { pub[0] = (uint32_t)(b0 + e); pub[1] = rem - above; pub[2] = hb[e]; }
                above += hb[e];
            }
        }
        lds_barrier();
        base += pub[0] << sh;
        span = min(span - (pub[0] << sh), sh ? (1u << sh) - 1u : 0u);
        rem = pub[1];
        if (sh == 0) break;                                // single keys: the threshold is base
        if (pub[2] <= FEW) {                               // (once: the loop ends here)
            const int n = (int)pub[2];
            each([&](int, uint32_t k) { if (k >= base && k - base <= span) few[atomicAdd(&nfew, 1u)] = k; });
            lds_barrier();
            // a wave compares every candidate, a lane each, with its share of them
            const uint32_t k = lane < n ? few[lane] : 0u;
            uint32_t c = 0u;                               // candidates above, and from bit 16 equal ones
            for (int e = wv; e < n; e += NW) {
                const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)k, e);
                c += o > k ? 1u : (o == k ? 0x10000u : 0u);
            }
            if (c) atomicAdd(&cmp[lane], c);
            lds_barrier();
            const uint32_t gt = cmp[lane] & 0xffffu, ge = gt + (cmp[lane] >> 16);
            const int l = (int)__builtin_ctzll(__ballot(lane < n && gt < rem && ge >= rem));   // (rem of the n are needed: never empty)
            base = (uint32_t)__builtin_amdgcn_readlane((int)k, l);
            rem -= (uint32_t)__builtin_amdgcn_readlane((int)gt, l);
            break;
        }
    }
    // taken: above the threshold, or equal to it while the equal ones before are fewer than rem
    uint32_t eq = 0u, gt = 0u, tot;
    each([&](int, uint32_t k) { eq += k == base ? 1u : 0u; gt += k > base ? 1u : 0u; });
    uint32_t before = block_excl<NW>(eq, tot, sc[0]);
    uint32_t pos = block_excl<NW>(gt + min(eq, rem > before ? rem - before : 0u), tot, sc[1]);
    each([&](int e, uint32_t k) {
        const bool t = k > base || (k == base && before < rem);
        before += k == base ? 1u : 0u;
        if (t) dst[pos++] = i0 + e;
    });
}

}  // namespace

hipError_t launch_quant_select(const QCache &q, int block, int dtype, const uint16_t *query, int num, int den, float *scores,
                               int32_t *list, hipStream_t s) {
    const int pairs = q.S * q.H;
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
