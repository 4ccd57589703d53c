// quant.h -- shared by the kernels of the 8-bit KV cache (quant_append.hip,
// quant_attn.h, quant_select.hip) and by their entry points (quant_api.hip)
// (not part of the C ABI).
#pragma once
#include "decode_common.h"

namespace mosaic {

constexpr float QLEAST = 7.888609052210118e-31f;          // 2^-100: magnitudes below count as this in a scale
constexpr int QF_E4M3 = 0, QF_INT8 = 1;
__host__ __device__ constexpr float q_top(int fmt) { return fmt == QF_INT8 ? 127.0f : 448.0f; }

constexpr int Q_ARRIVALS = 32;                             // a counter has a line of its own

// The cache's tensors (mosaic_quant_cache), passed by value.
struct QCache {
    int S, H, G, N;                                        // sequences, kv heads, group, blocks of a pair at most
    int cap;                                               // tokens of a sequence at most
    uint8_t *k, *v;                                        // codes [S][H][N][B][D] and [S][H][N][D][B]
    float *ks, *vs, *bs;                                   // scales of K, V and bounds [S][H][N]
    int8_t *bounds;                                        // [S][H][N][2][D]: upper, lower
    uint16_t *kt, *vt;                                     // unfinished block [S][H][B][D] and [S][H][D][B]
    int32_t *lens;                                         // [S][H]: a pair's workgroups need no other pair's
    int32_t *arrivals;                                     // [S][H][Q_ARRIVALS], the first of each used; zero between appends
    int32_t *refused;                                      // [S]: appends that a sequence had no room for
    // a pair's length; one that no append can have left reads as the nearest that can
    __device__ __forceinline__ int len(long long p) const { return min(max(lens[p], 0), cap); }
};

struct QNew {                                              // tokens to append, strides in elements
    const uint16_t *k, *v;
    int64_t k_seq, k_head, k_tok, v_seq, v_head, v_tok;
    const int32_t *counts;                                 // [S] on the device, or null: max_new each
    int max_new;
};

// How a launch shares the units of all pairs: in runs of c units that do not
// cross pairs, c the least that makes about `slots` runs, a multiple of step
// and at least cmin; from there up to 2 cmin for about `few` runs.  The lengths
// are read on the device, so a captured launch follows them; runs are equal
// however ragged the batch, and there are at most slots + pairs of them.
struct QShare {
    int slots, few, cmin, step;
    int least;                                             // runs of a pair at least
    int alone;                                             // units that a pair's only run may have, whatever c is
    int join;                                              // runs that are joined in one go: pairs of up to join * 2 cmin
                                                           // units have no more
};
struct QPlan {
    int s, h, i, ns;                                       // sequence, kv head, run of the pair, runs of the pair
    int c, L;                                              // units of a run, the sequence's tokens
    bool live;
};

// The plan of run w; units(L): units of a pair of L tokens.
template <typename U>
__device__ __forceinline__ QPlan q_plan(const QCache &q, const QShare &sh, U units, int w) {
    const int lane = threadIdx.x & 63;
    auto length = [&](int s) { return s < q.S ? q.len((long long)s * q.H) : 0; };
    const int L0 = length(lane);
    uint32_t total = lane < q.S ? (uint32_t)units(L0) : 0u;
    for (int s = lane + 64; s < q.S; s += 64) total += (uint32_t)units(length(s));
    total = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(total), 63) * (uint32_t)q.H;
    auto runs_of = [&](int n) { return (int)((total + (uint32_t)(n * sh.step) - 1u) / (uint32_t)(n * sh.step)) * sh.step; };
    const int c = max(max(sh.cmin, min(2 * sh.cmin, runs_of(sh.few))), runs_of(sh.slots));
    QPlan p{};
    uint32_t base = 0;
    for (int s0 = 0; s0 < q.S; s0 += 64) {
        const int s = s0 + lane, L = s0 ? length(s) : L0;
        const int u = s < q.S ? units(L) : 0;
        int cu = u <= sh.alone ? max(c, sh.alone) : c;
        if (u > sh.join * c && u <= sh.join * 2 * sh.cmin) cu = (u + sh.join * sh.step - 1) / (sh.join * sh.step) * sh.step;
        const int ns = s < q.S ? max(sh.least, (u + cu - 1) / cu) : 0;
        const uint32_t inc = wave_scan_add((uint32_t)(ns * q.H));
        const uint64_t hit = __ballot(base + inc > (uint32_t)w);       // the first sequence whose runs end past w
        if (hit) {
            const int l = (int)__builtin_ctzll(hit);
            p.s = s0 + l;
            p.ns = __builtin_amdgcn_readlane(ns, l);
            p.c = __builtin_amdgcn_readlane(cu, l);
            p.L = __builtin_amdgcn_readlane(L, l);
            const int r = w - ((int)(base + (uint32_t)__builtin_amdgcn_readlane((int)inc, l)) - p.ns * q.H);
            p.h = r / p.ns;
            p.i = r - p.h * p.ns;
            p.live = true;
            return p;
        }
        base += (uint32_t)__builtin_amdgcn_readlane((int)inc, 63);
    }
    return p;
}

// blocks of a pair of L tokens that a selection takes
__host__ __device__ __forceinline__ int q_want(int whole, int num, int den) {
    const long long n = ((long long)whole * num + den - 1) / den;
    return (int)(n < 1 ? (whole < 1 ? whole : 1) : (n > whole ? whole : n));
}

struct QSel {                                              // a selection, or list = null: every block
    int num, den;
    const int32_t *list;                                   // [pairs][N] ascending
};

// ---------------------------------------------------------------- launchers
hipError_t launch_quant_append(const QCache &q, int fmt, int block, int dtype, const QNew &n, hipStream_t s);
constexpr int Q_PAIRS = 64512;                             // pairs at most, and runs
constexpr int Q_RUNS = 65536;
// the attention's workspace: arrivals at pairs and at groups of runs [2][Q_RUNS]
// (zero between calls), then partials
size_t quant_attn_ws_bytes(int pairs);
hipError_t launch_quant_attn_e4m3(const QCache &q, int block, int dtype, const uint16_t *query, float scale, const QSel &sel,
                                  void *ws, float *out, hipStream_t s);
hipError_t launch_quant_attn_int8(const QCache &q, int block, int dtype, const uint16_t *query, float scale, const QSel &sel,
                                  void *ws, float *out, hipStream_t s);
// scores: [pairs][q_score_stride(N)]
__host__ __device__ __forceinline__ int q_score_stride(int n) { return (n + 3) & ~3; }
hipError_t launch_quant_select(const QCache &q, int block, int dtype, const uint16_t *query, int num, int den, float *scores,
                               int32_t *list, hipStream_t s);

}  // namespace mosaic
