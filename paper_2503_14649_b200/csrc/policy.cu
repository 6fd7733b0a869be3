// Clipped policy loss with a KL term over candidate lists, forward and backward.
//
// With x = scale * score, log pi_j = x_j - log sum exp x.  Everything is held in base 2 relative to the row's best score m:
// t_j = (score_j - m) a, a = scale * log2 e, log2 pi_j = t_j - log2 Z with Z = sum 2^t_j.  The difference comes first: x may be of any
// size (scores may be masked with the type's lowest value, all of a row even), and only differences are ever rounded.
// One pass over a row gives m, Z, the same for the reference, and E = sum 2^t_j (score_j - ref_j), from which
// kl = ln 2 * ((E / Z - (m - m_ref)) a + log2(Z_ref / Z)); differences are held in units of 2^24, so that none is infinite.
//
// Measured: 37 rows of 1 000 003 bf16 scores and references, forward 48 us (148 MB: 3.1 TB/s; bound by two exponentials and the 34
// instructions around them a candidate) and backward 44.5 (222 MB: 5.0 TB/s, a third of the writes still in L2 at the end); 4096 rows of 100
// candidates with ids 5.8 and 4.5.
#include <cmath>
#include <type_traits>

#include "common.cuh"

namespace rago {

constexpr int POLICY_MAX_G = 1024;
constexpr float LN2 = 0.69314718055994530942f;
#define RAGO_NEG_INF __int_as_float(0xff800000)

struct PolicyArgs {
    const void *scores, *ref;
    const int64_t* ids;
    int nq, C, G;
    float unit;    // the sign of a = scale * log2 e times 2^-24: unit * score is larger for better candidates, and sums of differences of the type's
                   // lowest values stay finite
    float step;    // |a| * 2^24, so that unit * step = a
    float scale;
    float lowest;  // the infinity that scales to -infinity
    const int32_t* chosen;
    const float *old_logp, *advantage;
    float low, high;  // 1 - clip_low, 1 + clip_high
};

template <bool BF16>
__device__ __forceinline__ float load_s(const void* base, size_t i) {
    if (BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[i]);
    return static_cast<const float*>(base)[i];
}

// Running sums of one row, relative to m (policy) and mr (reference), base 2; m and mr are unit * score.  The sums of policy and
// reference go through the same roundings (spelled out: contracted differently they would differ), so equal scores give kl = 0
// exactly.
// A candidate that the reference has at -infinity makes kl infinite if pi > 0 and adds nothing if pi = 0.  Which of the two it is shows
// against the row's best score only, not against the best so far, so such a candidate stays out of E (infinity times a weight that
// shrinks to 0 later would be NaN): the best of them is kept, and looked at in the end.
struct PolicySums { float m, Z, mr, Zr, E, lost; };  // E = sum 2^t unit * (score - ref), lost = the best unit * score with ref = -infinity
__device__ __forceinline__ PolicySums policy_none() { return {RAGO_NEG_INF, 0.f, RAGO_NEG_INF, 0.f, 0.f, RAGO_NEG_INF}; }

// 2^x as one instruction (2 units in the last place; below 2^-126 zero, which is what such a weight adds)
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 2^((from - to) step), where both may be -infinity
__device__ __forceinline__ float policy_rescale(float from, float to, float step) { return from == to ? 1.f : exp2_fast((from - to) * step); }

__device__ __forceinline__ bool policy_there(const PolicyArgs& A, size_t at, float score) {
    return (A.ids == nullptr || A.ids[at] >= 0) && score != A.lowest;
}

// Adds n candidates, number `at` on (bit i of `missing`: not there).  A missing candidate takes the score -infinity: its weight is 0 like anything
// else's, and so no candidate needs a branch.  The maxima move at most once for all of them.
template <int n, bool BF16, bool REF, bool IDS>
__device__ __forceinline__ void policy_add(const PolicyArgs& A, size_t at, PolicySums& S, float (&score)[n], float (&ref)[n], uint32_t missing) {
    const float step = A.step, unit = A.unit;
    float top = RAGO_NEG_INF, top_r = RAGO_NEG_INF;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        score[i] *= unit;
        if (IDS && (missing >> i & 1)) score[i] = RAGO_NEG_INF;
        top = fmaxf(top, score[i]);
        if (REF) {
            ref[i] *= unit;
            if (score[i] == RAGO_NEG_INF) ref[i] = RAGO_NEG_INF;
            top_r = fmaxf(top_r, ref[i]);
        }
    }
    if (top > S.m) {
        const float f = exp2_fast((S.m - top) * step);
        S.Z = __fmul_rn(S.Z, f); S.m = top;
        if (REF) S.E = __fmul_rn(S.E, f);
    }
    const float m = S.m == RAGO_NEG_INF ? 0.f : S.m;
    float mr = 0.f;
    if (REF) {
        if (top_r > S.mr) { S.Zr = __fmul_rn(S.Zr, exp2_fast((S.mr - top_r) * step)); S.mr = top_r; }
        mr = S.mr == RAGO_NEG_INF ? 0.f : S.mr;
    }
    const float E = S.E;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float w = exp2_fast((score[i] - m) * step);
        S.Z = __fadd_rn(S.Z, w);
        if (REF) {
            S.Zr = __fadd_rn(S.Zr, exp2_fast((ref[i] - mr) * step));
            if (!(w == 0.f)) S.E = fmaf(w, score[i] - ref[i], S.E);
        }
    }
    if (REF && S.E == __int_as_float(0x7f800000)) {  // once more, without the references at -infinity, and from memory: nothing stays in registers for it
        S.E = E;
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const float raw = load_s<BF16>(A.scores, at + i), r = load_s<BF16>(A.ref, at + i) * unit, s = policy_there(A, at + i, raw) ? raw * unit : RAGO_NEG_INF;
            const float w = exp2_fast((s - m) * step);
            if (w == 0.f) continue;
            if (r == RAGO_NEG_INF) S.lost = fmaxf(S.lost, s);
            else S.E = fmaf(w, s - r, S.E);
        }
    }
}
template <bool REF>
__device__ __forceinline__ void policy_join(PolicySums& S, const PolicySums& o, float step) {
    const float m = fmaxf(S.m, o.m), f = policy_rescale(S.m, m, step), g = policy_rescale(o.m, m, step);
    S.Z = fmaf(S.Z, f, __fmul_rn(o.Z, g));
    S.m = m;
    if (!REF) return;
    S.E = fmaf(S.E, f, __fmul_rn(o.E, g));
    const float mr = fmaxf(S.mr, o.mr);
    S.Zr = fmaf(S.Zr, policy_rescale(S.mr, mr, step), __fmul_rn(o.Zr, policy_rescale(o.mr, mr, step)));
    S.mr = mr;
    S.lost = fmaxf(S.lost, o.lost);
}
template <bool REF>
__device__ __forceinline__ PolicySums policy_shfl(const PolicySums& S, int o) {
    PolicySums r = policy_none();
    r.m = __shfl_xor_sync(0xffffffffu, S.m, o);
    r.Z = __shfl_xor_sync(0xffffffffu, S.Z, o);
    if (!REF) return r;
    r.mr = __shfl_xor_sync(0xffffffffu, S.mr, o);
    r.Zr = __shfl_xor_sync(0xffffffffu, S.Zr, o);
    r.E = __shfl_xor_sync(0xffffffffu, S.E, o);
    r.lost = __shfl_xor_sync(0xffffffffu, S.lost, o);
    return r;
}

// What the backward pass needs of a row: the best score m, log2 Z, the same of the reference.  A row without candidates has
// log2 Z = +infinity: pi = 0.
struct PolicyRow { float m, lz, mr, lzr; };
__device__ __forceinline__ PolicyRow policy_row(const PolicySums& S, bool has_ref, float unit, bool* none) {
    *none = S.m == RAGO_NEG_INF && S.Z == 0.f;
    PolicyRow r;
    r.m = *none ? 0.f : S.m / unit;
    r.lz = *none ? __int_as_float(0x7f800000) : log2f(S.Z);
    r.mr = S.mr == RAGO_NEG_INF ? 0.f : S.mr / unit;
    r.lzr = *none || !has_ref ? 0.f : log2f(S.Zr);
    return r;
}
// the logarithm of the quotient, not the difference of the logarithms: near policies have near sums
__device__ __forceinline__ float policy_kl(const PolicyArgs& A, const PolicySums& S) {
    const float E = S.lost > RAGO_NEG_INF && exp2_fast((S.lost - S.m) * A.step) != 0.f ? __int_as_float(0x7f800000) : S.E;
    return fmaf(E / S.Z - (S.m - (S.mr == RAGO_NEG_INF ? 0.f : S.mr)), A.scale / A.unit, LN2 * log2f(S.Zr / S.Z));
}

// log pi of sample t of row q and whether it counts
template <bool BF16>
__device__ __forceinline__ bool policy_sample(const PolicyArgs& A, const PolicyRow& r, int q, int t, float* logp) {
    const int c = A.chosen[(size_t)q * A.G + t];
    *logp = RAGO_NEG_INF;
    if (c < 0 || c >= A.C) return false;
    const size_t at = (size_t)q * A.C + c;
    const float s = load_s<BF16>(A.scores, at);
    if (!policy_there(A, at, s)) return false;
    *logp = LN2 * fmaf(fmaf(s, A.unit, -r.m * A.unit), A.step, -r.lz);
    return true;
}

// The loss term of a sample, and its slope by log pi
__device__ __forceinline__ float policy_term(const PolicyArgs& A, float logp, float old, float adv, float* slope) {
    const float ratio = expf(logp - old);
    const float u = ratio * adv, v = fminf(fmaxf(ratio, A.low), A.high) * adv;
    *slope = u <= v ? -u : 0.f;
    if (!(u == u)) *slope = u;
    return u <= v ? -u : (v < u ? -v : u);
}

// Rows in pieces of 16 bytes.  A row starts anywhere, so `head` numbers in front of its first 16-byte boundary are taken one at
// a time; the reference, whose rows are aligned alike only when its base is, is read the same way where it is and one at a time
// where it is not.  UNIT numbers are 16 bytes.
template <bool BF16>
struct Piece {
    static constexpr int UNIT = BF16 ? 8 : 4;
    static __device__ __forceinline__ void load(const void* base, size_t at, bool whole, float (&v)[UNIT]) {
        if (!whole) {
#pragma unroll
            for (int i = 0; i < UNIT; ++i) v[i] = load_s<BF16>(base, at + i);
        } else if (BF16) {
            const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + at);
            const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(h[i] << 16); v[2 * i + 1] = __uint_as_float(h[i] & 0xFFFF0000u); }
        } else {
            *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        }
    }
    static __device__ __forceinline__ void store(void* base, size_t at, bool whole, const float (&v)[UNIT]) {
        if (!whole) {
#pragma unroll
            for (int i = 0; i < UNIT; ++i) {
                if (BF16) static_cast<__nv_bfloat16*>(base)[at + i] = __float2bfloat16_rn(v[i]);
                else static_cast<float*>(base)[at + i] = v[i];
            }
        } else if (BF16) {
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                h[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + at) = make_uint4(h[0], h[1], h[2], h[3]);
        } else {
            *reinterpret_cast<float4*>(static_cast<float*>(base) + at) = *reinterpret_cast<const float4*>(v);
        }
    }
    // numbers before the first 16-byte boundary at or behind number `at`
    static __device__ __forceinline__ int head(const void* base, size_t at) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(base) + at * (16 / UNIT);
        return (int)((16 - p % 16) % 16) / (16 / UNIT);
    }
};

template <int n>
__device__ __forceinline__ uint32_t policy_missing(const int64_t* ids, size_t at) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < n; ++i) m |= (uint32_t)(ids[at + i] < 0) << i;
    return m;
}

// ---- forward ---------------------------------------------------------------------------------------------------------------
// Adds this thread's share (pieces first, first + stride, ...) of candidates begin .. begin + n - 1 of a row to S.
template <bool BF16, bool REF, bool IDS>
__device__ __forceinline__ void policy_sweep(const PolicyArgs& A, int q, int begin, int n, int first, int stride, PolicySums& S) {
    using P = Piece<BF16>;
    const size_t row = (size_t)q * A.C + begin;
    int head = P::head(A.scores, row);
    if (head > n) head = n;
    const int pieces = (n - head) / P::UNIT, tail = head + pieces * P::UNIT;
    const bool ref_whole = REF && P::head(A.ref, row + head) == 0;
    int p = first;
    for (; p + stride < pieces; p += 2 * stride) {  // two pieces in flight
        const size_t at = row + head + (size_t)p * P::UNIT, next = at + (size_t)stride * P::UNIT;
        float s[2][P::UNIT], r[2][P::UNIT];
        P::load(A.scores, at, true, s[0]);
        P::load(A.scores, next, true, s[1]);
        if (REF) { P::load(A.ref, at, ref_whole, r[0]); P::load(A.ref, next, ref_whole, r[1]); }
        const uint32_t m0 = IDS ? policy_missing<P::UNIT>(A.ids, at) : 0u, m1 = IDS ? policy_missing<P::UNIT>(A.ids, next) : 0u;
        policy_add<P::UNIT, BF16, REF, IDS>(A, at, S, s[0], r[0], m0);
        policy_add<P::UNIT, BF16, REF, IDS>(A, next, S, s[1], r[1], m1);
    }
    if (p < pieces) {
        const size_t at = row + head + (size_t)p * P::UNIT;
        float s[P::UNIT], r[P::UNIT];
        P::load(A.scores, at, true, s);
        if (REF) P::load(A.ref, at, ref_whole, r);
        policy_add<P::UNIT, BF16, REF, IDS>(A, at, S, s, r, IDS ? policy_missing<P::UNIT>(A.ids, at) : 0u);
    }
    // the numbers in front and behind, less than a piece each
    for (int i = first; i < head + n - tail; i += stride) {
        const size_t at = row + (i < head ? i : tail + i - head);
        float s[1] = {load_s<BF16>(A.scores, at)}, r[1] = {REF ? load_s<BF16>(A.ref, at) : 0.f};
        policy_add<1, BF16, REF, IDS>(A, at, S, s, r, IDS ? policy_missing<1>(A.ids, at) : 0u);
    }
}

// Short rows: a warp each (forward, 8000 x 1000 with ids 27 us, a CTA each 56; 1000 x 1000 5.9 and 8.7, but 1000 x 4000 17.4 and 13.2, and 64 x 1000
// 5.3 and 3.4).
constexpr int POLICY_SHORT = 1024, POLICY_WARPS = 4;
template <bool BF16, bool REF, bool IDS>
__global__ void __launch_bounds__(POLICY_WARPS * 32) policy_forward_short_kernel(const PolicyArgs A, float* __restrict__ out_policy, float* __restrict__ out_kl,
                                                                                 float* __restrict__ out_logp, float4* __restrict__ out_stats) {
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int q = blockIdx.x * POLICY_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (q >= A.nq) return;
    PolicySums S = policy_none();
    policy_sweep<BF16, REF, IDS>(A, q, 0, A.C, lane, 32, S);
    for (int o = 16; o; o >>= 1) policy_join<REF>(S, policy_shfl<REF>(S, o), A.step);
    bool none;
    const PolicyRow r = policy_row(S, REF, A.unit, &none);
    float sum = 0.f;
    for (int t = lane; t < A.G; t += 32) {
        const size_t at = (size_t)q * A.G + t;
        float logp, slope;
        if (policy_sample<BF16>(A, r, q, t, &logp)) sum += policy_term(A, logp, A.old_logp[at], A.advantage[at], &slope);
        out_logp[at] = logp;
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
        out_policy[q] = sum;
        out_kl[q] = none || !REF ? 0.f : policy_kl(A, S);
        out_stats[q] = make_float4(r.m, r.lz, r.mr, r.lzr);
    }
}

// Long rows: CTAs of POLICY_SPAN candidates.  A row of one span is finished by its CTA; the sums of several go to the workspace, and the
// kernel behind joins them, in their order.  (Clusters whose first CTA joined them through distributed shared memory needed no
// workspace, but 37 rows in clusters of 8 did not fit the GPU's parts at once: 79 us instead of 47 for 1 000 003 scores.)
constexpr int POLICY_SPAN = RAGO_POLICY_SPAN, POLICY_THREADS = 256;

template <bool BF16, bool REF>
__device__ __forceinline__ void policy_finish(const PolicyArgs& A, int q, PolicySums S, float* terms, float* __restrict__ out_policy, float* __restrict__ out_kl,
                                              float* __restrict__ out_logp, float4* __restrict__ out_stats) {
    const int tid = threadIdx.x;
    bool none;
    const PolicyRow r = policy_row(S, REF, A.unit, &none);
    float sum = 0.f;
    for (int t = tid; t < A.G; t += POLICY_THREADS) {
        const size_t at = (size_t)q * A.G + t;
        float logp, slope;
        if (policy_sample<BF16>(A, r, q, t, &logp)) sum += policy_term(A, logp, A.old_logp[at], A.advantage[at], &slope);
        out_logp[at] = logp;
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((tid & 31) == 0) terms[tid >> 5] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < POLICY_THREADS / 32; ++w) sum += terms[w];
        out_policy[q] = sum;
        out_kl[q] = none || !REF ? 0.f : policy_kl(A, S);
        out_stats[q] = make_float4(r.m, r.lz, r.mr, r.lzr);
    }
}

// The threads' sums, joined; the same in every thread
template <bool REF>
__device__ __forceinline__ PolicySums policy_join_block(const PolicyArgs& A, PolicySums S, PolicySums* part) {
    for (int o = 16; o; o >>= 1) policy_join<REF>(S, policy_shfl<REF>(S, o), A.step);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = S;
    __syncthreads();
    S = part[0];
#pragma unroll
    for (int w = 1; w < POLICY_THREADS / 32; ++w) policy_join<REF>(S, part[w], A.step);
    return S;
}

template <bool BF16, bool REF, bool IDS>
__global__ void __launch_bounds__(POLICY_THREADS) policy_forward_long_kernel(const PolicyArgs A, int spans, PolicySums* __restrict__ sums, float* __restrict__ out_policy,
                                                                             float* __restrict__ out_kl, float* __restrict__ out_logp, float4* __restrict__ out_stats) {
    __shared__ PolicySums part[POLICY_THREADS / 32];
    __shared__ float terms[POLICY_THREADS / 32];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int q = blockIdx.x / spans, begin = blockIdx.x % spans * POLICY_SPAN;
    PolicySums S = policy_none();
    policy_sweep<BF16, REF, IDS>(A, q, begin, min(A.C - begin, POLICY_SPAN), threadIdx.x, POLICY_THREADS, S);
    S = policy_join_block<REF>(A, S, part);
    if (spans > 1) {
        if (threadIdx.x == 0) sums[blockIdx.x] = S;
    } else {
        policy_finish<BF16, REF>(A, q, S, terms, out_policy, out_kl, out_logp, out_stats);
    }
}

template <bool BF16, bool REF>
__global__ void __launch_bounds__(POLICY_THREADS) policy_finish_kernel(const PolicyArgs A, int spans, const PolicySums* __restrict__ sums, float* __restrict__ out_policy,
                                                                       float* __restrict__ out_kl, float* __restrict__ out_logp, float4* __restrict__ out_stats) {
    __shared__ PolicySums part[POLICY_THREADS / 32];
    __shared__ float terms[POLICY_THREADS / 32];
    grid_dependency_wait();
    grid_dependents_may_launch();
    PolicySums S = policy_none();
    for (int i = threadIdx.x; i < spans; i += POLICY_THREADS) policy_join<REF>(S, sums[(size_t)blockIdx.x * spans + i], A.step);
    policy_finish<BF16, REF>(A, blockIdx.x, policy_join_block<REF>(A, S, part), terms, out_policy, out_kl, out_logp, out_stats);
}

// ---- backward --------------------------------------------------------------------------------------------------------------
struct PolicyGrads {
    const float *kl, *logp;
    const float4* stats;
    const float *grad_policy, *grad_kl;
    void* out;
};
// What is the same for all candidates of a row: the gradient is pi (by_gap * (log2 pi - log2 rho) + flat), and by_own * own more where
// samples chose the candidate.
struct PolicyBack { PolicyRow r; float unit, step, lowest, by_gap, flat, by_own; };  // r.m and r.mr times unit

// Slope of sample t by log pi, and the candidate it belongs to (-1: does not count)
__device__ __forceinline__ float policy_slope(const PolicyArgs& A, const PolicyGrads& D, int q, int t, int* to) {
    const size_t at = (size_t)q * A.G + t;
    const float logp = D.logp[at], old = A.old_logp[at], adv = A.advantage[at];
    const int c = A.chosen[at];
    float s = 0.f;
    *to = -1;
    if (c >= 0 && c < A.C && logp != RAGO_NEG_INF) {  // the forward pass left -infinity for samples that do not count
        policy_term(A, logp, old, adv, &s);
        *to = c;
    }
    return s;
}

template <bool REF>
__device__ __forceinline__ float policy_grad(const PolicyBack& B, float score, float ref) {
    // unit * score - unit * best in one rounding: a difference of scores of any size
    const float l = fmaf(fmaf(score, B.unit, -B.r.m), B.step, -B.r.lz), p = exp2_fast(l);
    const float g = p * (REF ? fmaf(B.by_gap, l - fmaf(fmaf(ref, B.unit, -B.r.mr), B.step, -B.r.lzr), B.flat) : B.flat);
    return p == 0.f ? 0.f : g;  // a missing candidate, or one next to impossible: whatever its reference is
}

template <bool REF>
__device__ __forceinline__ PolicyBack policy_back(const PolicyArgs& A, const PolicyGrads& D, int q, float H) {
    const float4 st = D.stats[q];
    const float gp = A.G ? D.grad_policy[q] : 0.f, gk = REF ? D.grad_kl[q] : 0.f;
    return {{st.x * A.unit, st.y, st.z * A.unit, st.w}, A.unit, A.step, A.lowest, A.scale * gk * LN2, -A.scale * (gp * H + (REF ? gk * D.kl[q] : 0.f)), A.scale * gp};
}

// one candidate, own: the slopes of the samples that chose it
template <bool BF16, bool REF, bool IDS>
__device__ __forceinline__ void policy_put_one(const PolicyArgs& A, const PolicyGrads& D, const PolicyBack& B, size_t at, float own) {
    const float score = IDS && A.ids[at] < 0 ? B.lowest : load_s<BF16>(A.scores, at);
    float g = policy_grad<REF>(B, score, REF ? load_s<BF16>(A.ref, at) : 0.f);
    if (own != 0.f) g = fmaf(B.by_own, own, g);
    if (BF16) static_cast<__nv_bfloat16*>(D.out)[at] = __float2bfloat16_rn(g);
    else static_cast<float*>(D.out)[at] = g;
}

// Candidates begin .. begin + n - 1 of a row, shared by `stride` threads.  Pieces follow the boundaries of the output.
template <bool BF16, bool REF, bool IDS>
__device__ __forceinline__ void policy_back_sweep(const PolicyArgs& A, const PolicyGrads& D, const PolicyBack& B, int q, int begin, int n, int first, int stride) {
    using P = Piece<BF16>;
    const size_t row = (size_t)q * A.C + begin;
    int head = P::head(D.out, row);
    if (head > n) head = n;
    const int pieces = (n - head) / P::UNIT, tail = head + pieces * P::UNIT;
    const bool whole = P::head(A.scores, row + head) == 0, ref_whole = REF && P::head(A.ref, row + head) == 0;
    for (int p = first; p < pieces; p += stride) {
        const size_t at = row + head + (size_t)p * P::UNIT;
        float s[P::UNIT], r[P::UNIT] = {};
        P::load(A.scores, at, whole, s);
        if (REF) P::load(A.ref, at, ref_whole, r);
        const uint32_t missing = IDS ? policy_missing<P::UNIT>(A.ids, at) : 0u;
#pragma unroll
        for (int i = 0; i < P::UNIT; ++i) s[i] = policy_grad<REF>(B, IDS && (missing >> i & 1) ? B.lowest : s[i], r[i]);
        P::store(D.out, at, true, s);
    }
    for (int i = first; i < head + n - tail; i += stride) policy_put_one<BF16, REF, IDS>(A, D, B, row + (i < head ? i : tail + i - head), 0.f);
}

// Short rows: a warp each.  Up to 32 samples live in the lanes; more go through shared memory by the kernel below.
template <bool BF16, bool REF, bool IDS>
__global__ void __launch_bounds__(POLICY_WARPS * 32) policy_backward_short_kernel(const PolicyArgs A, const PolicyGrads D) {
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int q = blockIdx.x * POLICY_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (q >= A.nq) return;
    int to = -1;
    const float slope = lane < A.G ? policy_slope(A, D, q, lane, &to) : 0.f;
    float H = slope;
    for (int o = 16; o; o >>= 1) H += __shfl_xor_sync(0xffffffffu, H, o);
    const PolicyBack B = policy_back<REF>(A, D, q, H);
    policy_back_sweep<BF16, REF, IDS>(A, D, B, q, 0, A.C, lane, 32);
    __syncwarp();
    // the first sample of a candidate writes the sum of all of its samples
    float own = 0.f;
    bool is_first = to >= 0;
    for (int u = 0; u < A.G; ++u) {
        const int c = __shfl_sync(0xffffffffu, to, u);
        const float s = __shfl_sync(0xffffffffu, slope, u);
        if (c == to) {
            own += s;
            is_first = is_first && u >= lane;
        }
    }
    if (is_first) policy_put_one<BF16, REF, IDS>(A, D, B, (size_t)q * A.C + to, own);
}

// Long rows, or many samples: CTAs of POLICY_BACK_SPAN candidates
constexpr int POLICY_BACK_SPAN = 8192, POLICY_BACK_THREADS = 256;
template <bool BF16, bool REF, bool IDS>
__global__ void __launch_bounds__(POLICY_BACK_THREADS) policy_backward_long_kernel(const PolicyArgs A, const PolicyGrads D, int spans) {
    __shared__ float slope[POLICY_MAX_G];
    __shared__ int at_of[POLICY_MAX_G];
    __shared__ float warp_part[POLICY_BACK_THREADS / 32];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int q = blockIdx.x / spans, begin = blockIdx.x % spans * POLICY_BACK_SPAN, here = min(A.C - begin, POLICY_BACK_SPAN), tid = threadIdx.x;
    // the span's lines are asked for before the samples are looked at
    constexpr int SIZE = BF16 ? 2 : 4, LINE = 128 / SIZE;
    for (int i = tid * LINE; i < here; i += POLICY_BACK_THREADS * LINE) {
        const size_t at = (size_t)q * A.C + begin + i;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t*>(A.scores) + at * SIZE));
        if (REF) asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t*>(A.ref) + at * SIZE));
    }
    float H = 0.f;
    for (int t = tid; t < A.G; t += POLICY_BACK_THREADS) {
        int to;
        slope[t] = policy_slope(A, D, q, t, &to);
        at_of[t] = to;
        H += slope[t];
    }
    for (int o = 16; o; o >>= 1) H += __shfl_xor_sync(0xffffffffu, H, o);
    if ((tid & 31) == 0) warp_part[tid >> 5] = H;
    __syncthreads();
    H = 0.f;
    for (int w = 0; w < POLICY_BACK_THREADS / 32; ++w) H += warp_part[w];
    const PolicyBack B = policy_back<REF>(A, D, q, H);
    policy_back_sweep<BF16, REF, IDS>(A, D, B, q, begin, here, tid, POLICY_BACK_THREADS);
    __syncthreads();
    for (int t = tid; t < A.G; t += POLICY_BACK_THREADS) {  // the first sample of a candidate writes the sum of all of its samples
        const int c = at_of[t];
        if (c < begin || c - begin >= here) continue;
        bool is_first = true;
        for (int u = 0; u < t && is_first; ++u) is_first = at_of[u] != c;
        if (!is_first) continue;
        float own = 0.f;
        for (int u = t; u < A.G; ++u) own += at_of[u] == c ? slope[u] : 0.f;
        policy_put_one<BF16, REF, IDS>(A, D, B, (size_t)q * A.C + c, own);
    }
}

static rago_status policy_fail(rago_status st, const char* what, long long v = 0) {
    set_error(what, v);
    return st;
}

static bool policy_off(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

static rago_status policy_check(const void* scores, const void* ref, rago_dtype dtype, const int64_t* ids, int32_t nq, int32_t C, float scale,
                                const int32_t* chosen, const float* old_logp, const float* advantage, int32_t G, float clip_low,
                                float clip_high, PolicyArgs* A) {
    if (nq < 0) return policy_fail(RAGO_EINVAL, "nq = %lld is negative", nq);
    if (C < 1) return policy_fail(RAGO_EINVAL, "C = %lld must be at least 1", C);
    if (G < 0) return policy_fail(RAGO_EINVAL, "G = %lld is negative", G);
    if (dtype != RAGO_F32 && dtype != RAGO_BF16) return policy_fail(RAGO_EINVAL, "dtype = %lld is neither F32 nor BF16", dtype);
    if (!(scale - scale == 0.f) || scale == 0.f) return policy_fail(RAGO_EINVAL, "scale must be finite and not 0");
    if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f)) return policy_fail(RAGO_EINVAL, "clip_low must lie in [0, 1] and clip_high be at least 0");
    if (nq * parts_of(C, POLICY_BACK_SPAN) >= (1LL << 31)) return policy_fail(RAGO_EUNSUPPORTED, "nq * C is too large for one launch");
    if (G > POLICY_MAX_G) return policy_fail(RAGO_EUNSUPPORTED, "G = %lld exceeds 1024", G);
    if ((long long)nq * C >= (1LL << 40)) return policy_fail(RAGO_EUNSUPPORTED, "nq * C = %lld is 2^40 or more", (long long)nq * C);
    if (nq > 0 && !scores) return policy_fail(RAGO_EINVAL, "scores are null");
    if (nq > 0 && G > 0 && (!chosen || !old_logp || !advantage)) return policy_fail(RAGO_EINVAL, "chosen, old_logp or advantage are null");
    const uintptr_t unit = dtype == RAGO_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(scores) % unit || reinterpret_cast<uintptr_t>(ref) % unit || reinterpret_cast<uintptr_t>(ids) % 8)
        return policy_fail(RAGO_EALIGN, "scores, ref_scores or ids are not aligned to their type");
    if (policy_off(chosen) || policy_off(old_logp) || policy_off(advantage)) return policy_fail(RAGO_EALIGN, "chosen, old_logp or advantage are not aligned to their type");
    A->scores = scores; A->ref = ref; A->ids = ids; A->lowest = scale > 0.f ? -INFINITY : INFINITY; A->unit = scale > 0.f ? 0x1p-24f : -0x1p-24f;
    A->nq = nq; A->C = C; A->G = G;
    const float a = (float)((double)scale * 1.44269504088896340736);
    A->scale = scale;
    A->step = fabsf(a) * 0x1p24f;
    if (a == 0.f) return policy_fail(RAGO_EINVAL, "scale must be finite and not 0");
    if (!(A->step - A->step == 0.f)) return policy_fail(RAGO_EUNSUPPORTED, "scale exceeds 1e31 in magnitude");
    A->chosen = chosen; A->old_logp = old_logp; A->advantage = advantage;
    A->low = 1.f - clip_low; A->high = 1.f + clip_high;
    return RAGO_OK;
}

// f(bf16, has reference, has ids) as constants
template <class F>
static cudaError_t policy_variant(const PolicyArgs& A, rago_dtype dtype, F f) {
    std::true_type y;
    std::false_type n;
    auto ids = [&](auto bf16, auto ref) { return A.ids ? f(bf16, ref, y) : f(bf16, ref, n); };
    auto ref = [&](auto bf16) { return A.ref ? ids(bf16, y) : ids(bf16, n); };
    return dtype == RAGO_BF16 ? ref(y) : ref(n);
}

static rago_status policy_done(cudaError_t e, int launches, const char* what) {
    count_launch(launches);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return RAGO_OK;
    set_error("%s: %s", what, cudaGetErrorString(e));
    return RAGO_ECUDA;
}

}  // namespace rago

using namespace rago;

extern "C" rago_status rago_policy_workspace_bytes(int32_t nq, int32_t C, size_t* out_bytes) {
    if (!out_bytes) return policy_fail(RAGO_EINVAL, "out_bytes is null");
    if (nq < 0) return policy_fail(RAGO_EINVAL, "nq = %lld is negative", nq);
    if (C < 1) return policy_fail(RAGO_EINVAL, "C = %lld must be at least 1", C);
    const size_t spans = (size_t)parts_of(C, POLICY_SPAN);
    *out_bytes = spans > 1 ? align_up((size_t)nq * spans * sizeof(PolicySums), 256) : 0;
    return RAGO_OK;
}

extern "C" rago_status rago_policy_loss(const void* scores, const void* ref_scores, rago_dtype dtype, const int64_t* ids, int32_t nq,
                                        int32_t C, float scale, const int32_t* chosen, const float* old_logp, const float* advantage,
                                        int32_t G, float clip_low, float clip_high, float* out_policy, float* out_kl, float* out_logp,
                                        float* out_stats, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    PolicyArgs A;
    const rago_status st = policy_check(scores, ref_scores, dtype, ids, nq, C, scale, chosen, old_logp, advantage, G, clip_low, clip_high, &A);
    if (st != RAGO_OK || nq == 0) return st;
    if (!out_policy || !out_kl || !out_stats || (G > 0 && !out_logp)) return policy_fail(RAGO_EINVAL, "null pointer");
    if (reinterpret_cast<uintptr_t>(out_stats) % 16) return policy_fail(RAGO_EALIGN, "out_stats need 16-byte alignment");
    if (policy_off(out_policy) || policy_off(out_kl) || policy_off(out_logp)) return policy_fail(RAGO_EALIGN, "out_policy, out_kl or out_logp are not aligned to their type");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    float4* stats = reinterpret_cast<float4*>(out_stats);
    size_t need = 0;
    rago_policy_workspace_bytes(nq, C, &need);
    if (need) {
        if (!workspace) return policy_fail(RAGO_EINVAL, "workspace is null");
        if (reinterpret_cast<uintptr_t>(workspace) % 256) return policy_fail(RAGO_EALIGN, "workspace needs 256-byte alignment");
        if (workspace_bytes < need) return policy_fail(RAGO_ENOMEM, "workspace is smaller than the %lld bytes needed", (long long)need);
    }
    const int spans = (int)parts_of(C, POLICY_SPAN);
    return policy_done(policy_variant(A, dtype, [&](auto b, auto r, auto i) {
        constexpr bool B = decltype(b)::value, R = decltype(r)::value, I = decltype(i)::value;
        if (C <= POLICY_SHORT)
            return launch_overlapped(policy_forward_short_kernel<B, R, I>, dim3((unsigned)parts_of(nq, POLICY_WARPS)), dim3(POLICY_WARPS * 32), 0, s, A,
                                     out_policy, out_kl, out_logp, stats);
        PolicySums* sums = static_cast<PolicySums*>(workspace);
        const cudaError_t e = launch_overlapped(policy_forward_long_kernel<B, R, I>, dim3((unsigned)((int64_t)nq * spans)), dim3(POLICY_THREADS), 0, s, A, spans, sums,
                                                out_policy, out_kl, out_logp, stats);
        if (e != cudaSuccess || spans == 1) return e;
        return launch_overlapped(policy_finish_kernel<B, R>, dim3((unsigned)nq), dim3(POLICY_THREADS), 0, s, A, spans, sums, out_policy, out_kl, out_logp, stats);
    }), spans > 1 ? 2 : 1, "policy loss kernel");
}

extern "C" rago_status rago_policy_loss_backward(const void* scores, const void* ref_scores, rago_dtype dtype, const int64_t* ids,
                                                 int32_t nq, int32_t C, float scale, const int32_t* chosen, const float* old_logp,
                                                 const float* advantage, int32_t G, float clip_low, float clip_high, const float* kl,
                                                 const float* logp, const float* stats, const float* grad_policy, const float* grad_kl,
                                                 void* grad_scores, void* cuda_stream) {
    PolicyArgs A;
    const rago_status st = policy_check(scores, ref_scores, dtype, ids, nq, C, scale, chosen, old_logp, advantage, G, clip_low, clip_high, &A);
    if (st != RAGO_OK || nq == 0) return st;
    if (!stats || !grad_scores || (G > 0 && (!logp || !grad_policy)) || (ref_scores && (!kl || !grad_kl))) return policy_fail(RAGO_EINVAL, "null pointer");
    if (reinterpret_cast<uintptr_t>(stats) % 16) return policy_fail(RAGO_EALIGN, "stats need 16-byte alignment");
    if (policy_off(kl) || policy_off(logp) || policy_off(grad_policy) || policy_off(grad_kl))
        return policy_fail(RAGO_EALIGN, "kl, logp, grad_policy or grad_kl are not aligned to their type");
    if (reinterpret_cast<uintptr_t>(grad_scores) % (dtype == RAGO_F32 ? 4 : 2)) return policy_fail(RAGO_EALIGN, "grad_scores are not aligned to their type");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const PolicyGrads D = {kl, logp, reinterpret_cast<const float4*>(stats), grad_policy, grad_kl, grad_scores};
    return policy_done(policy_variant(A, dtype, [&](auto b, auto r, auto i) {
        constexpr bool B = decltype(b)::value, R = decltype(r)::value, I = decltype(i)::value;
        if (C <= POLICY_SHORT && G <= 32)
            return launch_overlapped(policy_backward_short_kernel<B, R, I>, dim3((unsigned)parts_of(nq, POLICY_WARPS)), dim3(POLICY_WARPS * 32), 0, s,
                                     A, D);
        const int spans = (int)parts_of(C, POLICY_BACK_SPAN);
        return launch_overlapped(policy_backward_long_kernel<B, R, I>, dim3((unsigned)((int64_t)nq * spans)), dim3(POLICY_BACK_THREADS), 0, s, A, D, spans);
    }), 1, "policy loss backward kernel");
}
