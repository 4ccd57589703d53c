// quant_join.h -- how the waves of a workgroup and the runs of a pair of the
// caches' decode attentions are joined (quant_attn.h, quant4_attn.hip).
#pragma once
#include "quant.h"

namespace mosaic {

namespace {

constexpr int QA_NWV = 4;                                  // waves of a workgroup
constexpr int QA_HEADS = 8;
constexpr int QA_PART = QA_HEADS * (D + 2);                // floats of a partial: (max, sum) and averages of the heads

// partials, past the XCD's L2
__device__ __forceinline__ void put2(float *p, float2 x) {
    __hip_atomic_store((uint64_t *)p, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float *p) {
    return __builtin_bit_cast(float2, __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// ns partials, `stride` floats apart, joined: a thread takes four columns of
// every np-th one, np = 256 / (32 G) shares, joined in LDS; the loads of 8 are
// out together.  The result is that of threads [0, 32 G).
struct Joined { float M, S; float4 A; };
__device__ __forceinline__ Joined join_runs(const float *part, int stride, int ns, int G, float *lds) {
    constexpr int CB = 8;
    const int tid = threadIdx.x, cols = 32 * G, np = 64 * QA_NWV / cols;
    const int share = tid / cols, col = tid - share * cols, h = col >> 5;
    float M = -INFINITY, S = 0.0f;
    float4 A = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (share < np)
        for (int r0 = share; r0 < ns; r0 += CB * np) {
            float2 ml[CB], a[CB][2];
#pragma unroll
            for (int e = 0; e < CB; ++e) {
                const float *ps = part + (uint64_t)min(r0 + e * np, ns - 1) * stride;
                ml[e] = get2(ps + 2 * h);
                a[e][0] = get2(ps + 2 * QA_HEADS + 4 * col);
                a[e][1] = get2(ps + 2 * QA_HEADS + 4 * col + 2);
            }
            float mn = M;
#pragma unroll
            for (int e = 0; e < CB; ++e) {
                if (r0 + e * np >= ns) ml[e] = make_float2(-INFINITY, 0.0f);
                mn = fmaxf(mn, ml[e].x);
            }
            const float mb = mn == -INFINITY ? 0.0f : mn;
            S *= __builtin_amdgcn_exp2f(M - mb);
            M = mn;
            float s = S;
#pragma unroll
            for (int e = 0; e < CB; ++e) {
                ml[e].y *= __builtin_amdgcn_exp2f(ml[e].x - mb);
                s += ml[e].y;
            }
            const float inv = share_of(s), x = S * inv;
            A = make_float4(A.x * x, A.y * x, A.z * x, A.w * x);
            S = s;
#pragma unroll
            for (int e = 0; e < CB; ++e) {
                if (r0 + e * np >= ns) continue;
                const float y = ml[e].y * inv;
                A.x = fmaf(a[e][0].x, y, A.x);
                A.y = fmaf(a[e][0].y, y, A.y);
                A.z = fmaf(a[e][1].x, y, A.z);
                A.w = fmaf(a[e][1].y, y, A.w);
            }
        }
    float *x = lds + 8 * tid;
    if (share > 0 && share < np) {
        *(float4 *)x = A;
        x[4] = M;
        x[5] = S;
    }
    __syncthreads();
    if (share == 0)
        for (int e = 1; e < np; ++e) {
            const float *o = lds + 8 * (tid + e * cols);
            const float4 a = *(const float4 *)o;
            const float mn = fmaxf(M, o[4]), mb = mn == -INFINITY ? 0.0f : mn;
            float x = S * __builtin_amdgcn_exp2f(M - mb), y = o[5] * __builtin_amdgcn_exp2f(o[4] - mb);
            S = x + y;
            const float inv = share_of(S);
            x *= inv;
            y *= inv;
            A = make_float4(A.x * x + a.x * y, A.y * x + a.y * y, A.z * x + a.z * y, A.w * x + a.w * y);
            M = mn;
        }
    return Joined{M, S, A};
}

// Whether this workgroup is the last of n to arrive at a counter, which is zero
// again then.  What the workgroup wrote past the L2 can be read by the last
// one: every wave waits until its stores are acknowledged.  (A release fence in
// their place writes back the whole L2, 6 us a launch and more.)
__device__ __forceinline__ bool last_of(uint32_t *counter, int n, int &flag) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const bool l = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)n - 1u;
        if (l) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        flag = l;
    }
    __syncthreads();
    return flag;
}

// A compute unit reads partials at about 35 bytes a ns, so many runs are joined
// in groups first, by each group's last workgroup: runs of a group, 0 for none.
// (59 runs of 4 heads at once took 6.8 us; one sequence of one kv head has up to
// 511: 256 K tokens 38.4 us at once, 21 in groups.)
__device__ __forceinline__ int qa_group(int ns) { return ns <= 32 ? 0 : (ns <= 64 ? 8 : (ns <= 256 ? 16 : 32)); }

// what w's upper half, as bf16, leaves of it (`half`: its mask, or 0 for all of w)
__device__ __forceinline__ float beyond(float w, uint32_t half = 0xffff0000u) { return w - __uint_as_float(__float_as_uint(w) & half); }
// upper halves of eight values
__device__ __forceinline__ dbf8 upper_halves(const float (&x)[8]) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
    dbf8 r;
    __builtin_memcpy(&r, o, 16);
    return r;
}

// The end of a workgroup's run: its waves joined, and by the pair's last
// workgroup the runs.  mrg[wave][row]: rows h, GP + h (, 2 GP + h) are the NP parts
// of head h's sums from column 2 on; (row h, 0) its running maximum, (h, 1) the
// sum of its weights, (GP + h, 0) the unit of its sums and, with SHIFT, (GP + h,
// 1) what is added to each of its averages.
template <int GP, int NP, bool SHIFT>
__device__ __forceinline__ void join_waves(float (&mrg)[QA_NWV][16][D + 2], int &last, const QPlan &pl, int G, int p,
                                           uint32_t *arrivals, float *part, float *outp) {
    const int tid = threadIdx.x;
    __syncthreads();
    float *out = outp + (uint64_t)p * G * D;
    // partials of a pair's runs are consecutive: run 0's is this workgroup's less pl.i
    float *mine = part + (uint64_t)blockIdx.x * QA_PART;
    for (int i = 2 * tid; i < G * D; i += 128 * QA_NWV) {    // two columns of a head
        const int h = i / D, c = i % D;
        float m[QA_NWV], M = -INFINITY;
#pragma unroll
        for (int w = 0; w < QA_NWV; ++w) { m[w] = mrg[w][h][0]; M = fmaxf(M, m[w]); }
        float2 A = make_float2(0.0f, 0.0f);
        float f[QA_NWV], S = 0.0f;
#pragma unroll
        for (int w = 0; w < QA_NWV; ++w) {
            f[w] = m[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[w] - M);
            S += mrg[w][h][1] * f[w];
        }
        const float inv = share_of(S);
#pragma unroll
        for (int w = 0; w < QA_NWV; ++w) {
            const float fu = f[w] * inv * mrg[w][h + GP][0];
            float2 u = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int e = NP - 1; e >= 0; --e) {   // the parts, from the least
                const float2 v = *(const float2 *)&mrg[w][h + GP * e][2 + c];
                u.x += v.x;
                u.y += v.y;
            }
            const float add = SHIFT ? mrg[w][h + GP][1] * (f[w] * mrg[w][h][1] * inv) : 0.0f;
            A.x += SHIFT ? fmaf(u.x, fu, add) : u.x * fu;
            A.y += SHIFT ? fmaf(u.y, fu, add) : u.y * fu;
        }
        if (pl.ns == 1) {
            *(float2 *)(out + i) = A;
        } else {
            put2(mine + 2 * QA_HEADS + i, A);
            if (c == 0) put2(mine + 2 * h, make_float2(M, S));
        }
    }
    if (pl.ns == 1) return;
    // the last workgroup of a group, then of the pair, joins its runs, in their
    // order whichever it is; partials are written and read past the XCD's L2
    const float *first = part + (uint64_t)(blockIdx.x - pl.i) * QA_PART;
    const int group = qa_group(pl.ns);
    int ns = pl.ns, stride = QA_PART;
    if (group) {
        const int at = pl.i / group * group;
        if (!last_of(arrivals + Q_RUNS + (blockIdx.x - pl.i + at), min(group, ns - at), last)) return;
        const Joined j = join_runs(first + (uint64_t)at * QA_PART, QA_PART, min(group, ns - at), G, &mrg[0][0][0]);
        if (tid < 32 * G) {                              // to the place of the group's first run
            float *to = part + (uint64_t)(blockIdx.x - pl.i + at) * QA_PART;
            put2(to + 2 * QA_HEADS + 4 * tid, make_float2(j.A.x, j.A.y));
            put2(to + 2 * QA_HEADS + 4 * tid + 2, make_float2(j.A.z, j.A.w));
            if (tid % 32 == 0) put2(to + tid / 16, make_float2(j.M, j.S));
        }
        ns = (ns + group - 1) / group;
        stride = group * QA_PART;
    }
    if (!last_of(arrivals + p, ns, last)) return;
    const Joined j = join_runs(first, stride, ns, G, &mrg[0][0][0]);
    if (tid < 32 * G) *(float4 *)(out + 4 * tid) = j.A;
}

}  // namespace

}  // namespace mosaic
