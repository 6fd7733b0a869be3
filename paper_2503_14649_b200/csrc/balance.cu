// Probes counted per inverted list, and the balance loss of the coarse quantiser, forward and backward.
//
// loss = nlist / n * sum_rows sum_l f_l p_l with f_l = counts_l / T: given the counts, a row needs one pass for some logit m near
// its best, Z = sum 2^t_l and D = sum counts_l 2^t_l (t_l = (logit_l - m) a, a = scale * log2 e; the difference comes first, so logits may be
// of any size, masked with the type's lowest value among them); the mean of p over the batch is never formed.  The smallest count
// is taken off all counts first, exactly: what the gradient is made of, f_l less the row's sum f p, is then not lost where lists are
// nearly even, and 0 where they are.  The backward pass reads the logits once more and writes the gradient.
//
// Measured: 4096 rows of 65 536 bf16 logits, forward 128 to 138 us (537 MB: 3.9 to 4.2 TB/s; exponentials and the ten instructions around
// them) and backward 176 to 181 (1.07 GB: 6.0 TB/s), by the GPU at hand; 1021 rows of 4096 fp32 logits 18 and 6.3.
#include <type_traits>

#include "common.cuh"

namespace rago {

constexpr int BALANCE_THREADS = 256;

// What the rows leave for the backward pass, float4 per row: m, 1 / Z, sum f p less base / T, a word of the CTA's; row nq:
// nlist / n, 1 / T, and as whole numbers n, in whose place the last CTA leaves the base (what is taken off all counts), and T.  Until the last CTA has added the rows up, the word of nlist / n is the ticket by which it knows that it is the last.
struct BalanceTotals { float per_row, per_slot; uint32_t rows, slots; };

template <bool BF16>
__device__ __forceinline__ float load_l(const void* base, size_t i) {
    if (BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[i]);
    return static_cast<const float*>(base)[i];
}
// 2^x as one instruction (2 units in the last place; below 2^-126 zero, which is what such a weight adds)
__device__ __forceinline__ float balance_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- counts ------------------------------------------------------------------------------------------------------------------
// Whole numbers: the order of the additions does not matter.  Up to BALANCE_RANGE_SLOTS slots are read by every one of a few CTAs, each
// of which counts its range of lists in shared memory and writes it: one launch, nothing to clear.  (At 32 000 slots of 4096 lists
// that takes 2.4 us longer on the GPU than clearing and adding, which is captured calls' loss, and saves a launch of 4 us on the host, which
// bounds such calls otherwise; at 6400 slots of 65 536 lists it is 3 us faster on the GPU too.)  More slots are dealt out to CTAs, which add what they
// counted (in shared memory where the lists fit, so that few lists are not contended for) to counts that were cleared before.
constexpr int BALANCE_SHORT_LISTS = 1024;  // rows of up to as many are short: part of a warp each, or a warp
constexpr int BALANCE_OWN_LEAST = 4096;
constexpr int BALANCE_SHARED_LISTS = 8192, BALANCE_RANGE_SLOTS = 1 << 15, BALANCE_RANGE_LISTS = 1024, BALANCE_RANGE_CTAS = 64, BALANCE_COUNT_THREADS = 512;

// Lists l0 .. l0 + range - 1 per CTA; the first one also counts slots and rows
constexpr int BALANCE_RANGE_THREADS = 1024;
__global__ void __launch_bounds__(BALANCE_RANGE_THREADS) balance_count_ranges_kernel(const int32_t* __restrict__ lists, const uint8_t* __restrict__ valid, int nq,
                                                                                     int nprobe, int nlist, int range, int32_t* __restrict__ counts,
                                                                                     BalanceTotals* __restrict__ totals, uint32_t* __restrict__ ticket) {
    extern __shared__ int32_t here[];
    __shared__ uint32_t sums[2];
    const int tid = threadIdx.x, l0 = blockIdx.x * range, mine = nlist - l0 < range ? nlist - l0 : range;
    for (int l = tid; l < mine; l += BALANCE_RANGE_THREADS) here[l] = 0;
    if (tid < 2) sums[tid] = 0;
    __syncthreads();
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int all = nq * nprobe;
    uint32_t slots = 0, rows = 0;
    auto count = [&](int l) {
        slots += l >= 0 && l < nlist;
        if (l >= l0 && l - l0 < mine) atomicAdd(&here[l - l0], 1);
    };
    if (nprobe % 4 == 0 && reinterpret_cast<uintptr_t>(lists) % 16 == 0) {  // four slots of one row at a time
        const int4* four = reinterpret_cast<const int4*>(lists);
#pragma unroll 4
        for (int i = tid; i < all / 4; i += BALANCE_RANGE_THREADS) {
            const int4 l = four[i];
            if (valid && !valid[(uint32_t)i * 4u / (uint32_t)nprobe]) continue;
            count(l.x); count(l.y); count(l.z); count(l.w);
        }
    } else {
#pragma unroll 4
        for (int i = tid; i < all; i += BALANCE_RANGE_THREADS) {
            const int l = lists[i];
            if (valid && !valid[(uint32_t)i / (uint32_t)nprobe]) continue;
            count(l);
        }
    }
    if (blockIdx.x == 0) {
        if (valid)
            for (int q = tid; q < nq; q += BALANCE_RANGE_THREADS) rows += valid[q] != 0;
        else rows = tid == 0 ? nq : 0;
        slots = __reduce_add_sync(0xffffffffu, slots);
        rows = __reduce_add_sync(0xffffffffu, rows);
        if ((tid & 31) == 0) { atomicAdd(&sums[0], slots); atomicAdd(&sums[1], rows); }
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) { totals->slots = sums[0]; totals->rows = sums[1]; *ticket = 0u; }
    for (int l = tid; l < mine; l += BALANCE_RANGE_THREADS) counts[l0 + l] = here[l];
}

__global__ void __launch_bounds__(BALANCE_THREADS) balance_clear_kernel(int32_t* __restrict__ counts, int nlist, BalanceTotals* __restrict__ totals, uint32_t* __restrict__ ticket) {
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int i = blockIdx.x * BALANCE_THREADS + threadIdx.x;
    if (i < nlist) counts[i] = 0;
    if (i == 0) { totals->rows = totals->slots = 0u; *ticket = 0u; totals->per_slot = __int_as_float(0); }
}

// The smallest count, where the word that 1 / T goes to in the end holds it (volatile: read once, before the last CTA overwrites it)
__device__ __forceinline__ int balance_kept(const BalanceTotals* totals) { return __float_as_int(*const_cast<const volatile float*>(&totals->per_slot)); }
// The smallest of all counts, by a CTA.  A thread that has met a 0 is done.
template <int THREADS>
__device__ __forceinline__ int balance_least(const int32_t* counts, int nlist) {
    __shared__ int least;
    if (threadIdx.x == 0) least = 0x7fffffff;
    __syncthreads();
    int base = 0x7fffffff;
    const int whole = (reinterpret_cast<uintptr_t>(counts) & 15) == 0 ? nlist / 4 : 0;  // in fours
    for (int l = threadIdx.x; l < whole && base; l += 8 * THREADS) {
        int4 c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = reinterpret_cast<const int4*>(counts)[min(l + i * THREADS, whole - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) base = min(min(base, min(c[i].x, c[i].y)), min(c[i].z, c[i].w));
    }
    for (int64_t l = 4 * whole + threadIdx.x; l < nlist && base; l += THREADS) base = min(base, counts[l]);
    base = __reduce_min_sync(0xffffffffu, base);
    if ((threadIdx.x & 31) == 0) atomicMin(&least, base);
    __syncthreads();
    return least;
}

// How the CTAs of long rows come by the smallest count: it is 0 where there are fewer slots than lists, which the host knows
enum BalanceLeast { BALANCE_LEAST_0, BALANCE_LEAST_OWN, BALANCE_LEAST_KEPT };

// SHARED: count in shared memory.  Up to BALANCE_OWN_LEAST counts, which 128 threads read in one go, the rows' CTAs find the smallest
// themselves (0.8 us at 1021 rows of 4096 lists, 2.3 by the last CTA here); of more the last CTA here does (2.2 us at 4096 rows of
// 8192 lists, 4.9 by the rows' CTAs).
template <bool SHARED>
__global__ void __launch_bounds__(BALANCE_COUNT_THREADS) balance_count_kernel(const int32_t* __restrict__ lists, const uint8_t* __restrict__ valid, int nq,
                                                                              int nprobe, int nlist, bool find_least, int32_t* __restrict__ counts, BalanceTotals* __restrict__ totals) {
    extern __shared__ int32_t here[];
    const int tid = threadIdx.x;
    if (SHARED) {
        for (int l = tid; l < nlist; l += BALANCE_COUNT_THREADS) here[l] = 0;
        __syncthreads();
    }
    grid_dependency_wait();
    grid_dependents_may_launch();
    uint32_t slots = 0, rows = 0;
    const int64_t all = (int64_t)nq * nprobe;
    for (int64_t i = (int64_t)blockIdx.x * BALANCE_COUNT_THREADS + tid; i < all; i += (int64_t)gridDim.x * BALANCE_COUNT_THREADS) {
        const uint32_t q = (uint32_t)i / (uint32_t)nprobe;  // nq * nprobe < 2^31
        if (valid && !valid[q]) continue;
        rows += (uint32_t)i == q * (uint32_t)nprobe;
        const int l = lists[i];
        if (l < 0 || l >= nlist) continue;
        ++slots;
        atomicAdd(SHARED ? &here[l] : &counts[l], 1);
    }
    slots = __reduce_add_sync(0xffffffffu, slots);
    rows = __reduce_add_sync(0xffffffffu, rows);
    __shared__ uint32_t sums[2];
    if (tid < 2) sums[tid] = 0;
    __syncthreads();
    if ((tid & 31) == 0) { atomicAdd(&sums[0], slots); atomicAdd(&sums[1], rows); }
    __syncthreads();
    if (tid == 0) {
        atomicAdd(&totals->slots, sums[0]);
        atomicAdd(&totals->rows, sums[1]);
    }
    if (SHARED)
        for (int l = tid; l < nlist; l += BALANCE_COUNT_THREADS)
            if (here[l]) atomicAdd(&counts[l], here[l]);
    if (!find_least) return;
    // the word of 1 / T counts the CTAs that are done, and holds the smallest count from then on until the rows are done
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(reinterpret_cast<uint32_t*>(&totals->per_slot), 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int base = balance_least<BALANCE_COUNT_THREADS>(counts, nlist);
    if (tid == 0) totals->per_slot = __int_as_float(base);
}

// ---- rows --------------------------------------------------------------------------------------------------------------------
struct BalanceSums { float m, Z, D; };  // relative to the logit m, base 2; D of the counts less the base
// Nothing yet: m is the infinity that scales to -infinity
__device__ __forceinline__ BalanceSums balance_none(float a) { return {a > 0.f ? __int_as_float(0xff800000) : __int_as_float(0x7f800000), 0.f, 0.f}; }
__device__ __forceinline__ bool balance_set(float m, float a) { return m != (a > 0.f ? __int_as_float(0xff800000) : __int_as_float(0x7f800000)); }
__device__ __forceinline__ bool balance_better(float x, float than, float a) { return a > 0.f ? x > than : x < than; }
__device__ __forceinline__ void balance_join(BalanceSums& S, const BalanceSums& o, float a) {
    const float m = balance_better(o.m, S.m, a) ? o.m : S.m, f = S.m == m ? 1.f : balance_exp2((S.m - m) * a), g = o.m == m ? 1.f : balance_exp2((o.m - m) * a);
    S.Z = S.Z * f + o.Z * g;
    S.D = S.D * f + o.D * g;
    S.m = m;
}
// Adds n numbers.  m need not be the best, only near it: the weights are taken relative to it as it stands, and only where they come
// out large (or it is not set, which makes them infinite or NaN) is the best looked for, moved to, and the weights taken again.
// (That a difference is taken before it is scaled took the forward pass from 113 to 136 us at 4096 x 65 536; scaled first, with the maximum's rounding taken
// off in the end, it took as long: registers.)
constexpr float BALANCE_NEAR = 65536.f;
template <int n>
__device__ __forceinline__ void balance_weigh(const float (&logit)[n], const float (&count)[n], float a, float m, float& z, float& d) {
    z = d = 0.f;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float w = balance_exp2((logit[i] - m) * a);
        z += w;
        d = fmaf(w, count[i], d);
    }
}
template <int n>
__device__ __forceinline__ void balance_add(BalanceSums& S, const float (&logit)[n], const float (&count)[n], float a) {
    float z, d;
    balance_weigh<n>(logit, count, a, S.m, z, d);
    if (!(z < BALANCE_NEAR)) {
        float top = S.m;
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (balance_better(logit[i], top, a)) top = logit[i];
        if (top != S.m) {
            const float f = balance_exp2((S.m - top) * a);
            S.Z *= f; S.D *= f; S.m = top;
        }
        balance_weigh<n>(logit, count, a, balance_set(S.m, a) ? S.m : 0.f, z, d);
    }
    S.Z += z;
    S.D += d;
}

// 16 bytes of a row, aligned
template <bool BF16>
struct LogitPiece {
    static constexpr int UNIT = BF16 ? 8 : 4;
    static __device__ __forceinline__ uint4 load(const void* base, size_t at) {
        return __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(base) + at * (16 / UNIT)));
    }
    static __device__ __forceinline__ void values(const uint4& w, float (&v)[UNIT]) {
        const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (BF16) { v[2 * i] = __uint_as_float(h[i] << 16); v[(2 * i + 1) % UNIT] = __uint_as_float(h[i] & 0xFFFF0000u); }
            else v[i] = __uint_as_float(h[i]);
    }
    static __device__ __forceinline__ void store(void* base, size_t at, const float (&v)[UNIT]) {
        if (BF16) {
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                h[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
            __stcs(reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + at), make_uint4(h[0], h[1], h[2], h[3]));
        } else {
            __stcs(reinterpret_cast<float4*>(static_cast<float*>(base) + at), *reinterpret_cast<const float4*>(v));
        }
    }
    static __device__ __forceinline__ void counts(const int32_t* c, int l, int base, float (&v)[UNIT]) {
#pragma unroll
        for (int i = 0; i < UNIT; i += 4) {
            const int4 w = *reinterpret_cast<const int4*>(c + l + i);
            v[i] = (float)(w.x - base); v[i + 1] = (float)(w.y - base); v[i + 2] = (float)(w.z - base); v[i + 3] = (float)(w.w - base);
        }
    }
};

// Counts start .. start + UNIT - 1, less the base, as floats, from whole aligned words where they have neighbours to be cut out of
// (start & 3 is the same for all pieces of a row), one at a time else: eight separate loads a lane cost the L1 eight times what the
// logits do.
template <bool BF16>
__device__ __forceinline__ void balance_window(const int32_t* __restrict__ counts, int start, int nlist, int base, float (&v)[LogitPiece<BF16>::UNIT]) {
    constexpr int UNIT = LogitPiece<BF16>::UNIT;
    const int shift = start & 3;
    const bool aligned = (reinterpret_cast<uintptr_t>(counts) & 15) == 0;
    if (aligned && shift == 0) {
        LogitPiece<BF16>::counts(counts, start, base, v);
    } else if (aligned && start - shift <= nlist - (UNIT + 4)) {
        int w[UNIT + 4];
#pragma unroll
        for (int i = 0; i < UNIT + 4; i += 4) *reinterpret_cast<int4*>(w + i) = *reinterpret_cast<const int4*>(counts + start - shift + i);
        if (shift == 1) {
#pragma unroll
            for (int i = 0; i < UNIT; ++i) v[i] = (float)(w[i + 1] - base);
        } else if (shift == 2) {
#pragma unroll
            for (int i = 0; i < UNIT; ++i) v[i] = (float)(w[i + 2] - base);
        } else {
#pragma unroll
            for (int i = 0; i < UNIT; ++i) v[i] = (float)(w[i + 3] - base);
        }
    } else {
#pragma unroll
        for (int i = 0; i < UNIT; ++i) v[i] = (float)(counts[start + i] - base);
    }
}
// Numbers of a row in front of its first 16-byte boundary
template <bool BF16>
__device__ __forceinline__ int balance_head(const void* base, size_t row, int nlist) {
    constexpr int SIZE = BF16 ? 2 : 4;
    const int head = (int)((16 - (reinterpret_cast<uintptr_t>(base) + row * SIZE) % 16) % 16) / SIZE;
    return head < nlist ? head : nlist;
}

// A thread's share (pieces first, first + stride, ...) of one row.  A row may start anywhere: what lies in front of its first
// 16-byte boundary and behind its last is taken one number at a time, and the counts, which then lie across boundaries, too.
template <bool BF16>
__device__ __forceinline__ void balance_sweep(BalanceSums& S, const void* __restrict__ logits, size_t row, int nlist, float a, const int32_t* __restrict__ counts,
                                              int base, int first, int stride) {
    using P = LogitPiece<BF16>;
    const int head = balance_head<BF16>(logits, row, nlist), pieces = (nlist - head) / P::UNIT, tail = head + pieces * P::UNIT;
    uint4 next = make_uint4(0, 0, 0, 0);
    if (first < pieces) next = P::load(logits, row + head + (size_t)first * P::UNIT);
    for (int p = first; p < pieces; p += stride) {
        const uint4 w = next;  // the piece behind is on its way while this one is added
        if (p + stride < pieces) next = P::load(logits, row + head + (size_t)(p + stride) * P::UNIT);
        float c[P::UNIT], v[P::UNIT];
        balance_window<BF16>(counts, head + p * P::UNIT, nlist, base, c);
        P::values(w, v);
        balance_add<P::UNIT>(S, v, c, a);
    }
    for (int i = first; i < head + (nlist - tail); i += stride) {
        const int l = i < head ? i : tail + (i - head);
        const float v[1] = {load_l<BF16>(logits, row + l)}, c[1] = {(float)(counts[l] - base)};
        balance_add<1>(S, v, c, a);
    }
}

// over LANES neighbouring lanes
template <int LANES = 32>
__device__ __forceinline__ void balance_join_warp(BalanceSums& S, float a) {
    for (int o = LANES / 2; o; o >>= 1) {
        const BalanceSums other = {__shfl_xor_sync(0xffffffffu, S.m, o), __shfl_xor_sync(0xffffffffu, S.Z, o), __shfl_xor_sync(0xffffffffu, S.D, o)};
        balance_join(S, other, a);
    }
}

// m, 1 / Z, sum f p less base / T of a row; the last word is the CTA's
__device__ __forceinline__ float4 balance_stats(const BalanceSums& s, uint32_t T) {
    const bool none = s.Z == 0.f;
    const float inv = none ? 0.f : 1.f / s.Z;
    return make_float4(none ? 0.f : s.m, inv, none || !T ? 0.f : s.D * inv / (float)T, 0.f);
}

// After the CTA's rows (ROWS of them from q0 on, their stats in `mine`, in shared memory): their sum goes into the unused word of
// the first one's stats, and the last CTA to get here adds the CTAs' sums up, in their order.
template <int ROWS, int THREADS>
__device__ __forceinline__ void balance_close(const float4* mine, int q0, int nq, int nlist, uint32_t T, int base, BalanceTotals* __restrict__ totals, uint32_t* __restrict__ ticket,
                                              float4* __restrict__ stats, float* __restrict__ loss) {
    __shared__ float sums[THREADS / 32];
    __shared__ bool last;
    const int tid = threadIdx.x;
    __syncthreads();
    for (int r = tid; r < ROWS; r += THREADS)
        if (q0 + r < nq) {
            float4 st = mine[r];
            if (r == 0) {
                const float even = T ? (float)base / (float)T : 0.f;
                float sum = 0.f;
                for (int i = 0; i < ROWS; ++i)
                    if (q0 + i < nq && mine[i].y != 0.f) sum += even + mine[i].z;  // 1 / Z = 0: nothing in the row, or it is not counted
                st.w = sum;
            }
            stats[q0 + r] = st;
        }
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    float sum = 0.f;
#pragma unroll 8
    for (int i = tid; i < (int)gridDim.x; i += THREADS) sum += __ldcg(&stats[(size_t)i * ROWS].w);
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((tid & 31) == 0) sums[tid >> 5] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < THREADS / 32; ++w) sum += sums[w];
        const uint32_t n = totals->rows;
        const float per_row = n ? (float)nlist / (float)n : 0.f;
        totals->per_row = per_row;
        totals->per_slot = T ? 1.f / (float)T : 0.f;
        totals->rows = (uint32_t)base;
        *loss = per_row * sum;
    }
}

// Short rows: LANES lanes each, PASSES times one after the other
template <bool BF16, int LANES, int PASSES>
__global__ void __launch_bounds__(BALANCE_THREADS) balance_short_rows_kernel(const void* __restrict__ logits, int nq, int nlist, float a, const uint8_t* __restrict__ valid,
                                                                             const int32_t* __restrict__ counts, BalanceTotals* __restrict__ totals,
                                                                             uint32_t* __restrict__ ticket, float4* __restrict__ stats, float* __restrict__ loss) {
    constexpr int TEAMS = BALANCE_THREADS / LANES, ROWS = TEAMS * PASSES;
    __shared__ float4 mine[ROWS];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int q0 = blockIdx.x * ROWS, lane = threadIdx.x % LANES;
    const uint32_t T = totals->slots;
    __shared__ int least;
    if (threadIdx.x == 0) least = 0x7fffffff;
    __syncthreads();
    int base = 0x7fffffff;
    for (int l = threadIdx.x; l < nlist; l += BALANCE_THREADS) base = min(base, counts[l]);
    base = __reduce_min_sync(0xffffffffu, base);
    if ((threadIdx.x & 31) == 0) atomicMin(&least, base);
    __syncthreads();
    base = least;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        const int r = pass * TEAMS + threadIdx.x / LANES;
        BalanceSums S = balance_none(a);
        if (q0 + r < nq && (!valid || valid[q0 + r])) balance_sweep<BF16>(S, logits, (size_t)(q0 + r) * nlist, nlist, a, counts, base, lane, LANES);
        balance_join_warp<LANES>(S, a);
        if (lane == 0) mine[r] = balance_stats(S, T);
    }
    balance_close<ROWS, BALANCE_THREADS>(mine, q0, nq, nlist, T, base, totals, ticket, stats, loss);
}

// Long rows: ROWS of them per CTA, so that the counts, which come from L2 in twice the bytes of bf16 logits, are read once for all of
// them (WHOLE: rows and counts of whole 16-byte pieces), or are at least met again in L1.
template <bool BF16, int ROWS, bool WHOLE, int THREADS>
__global__ void __launch_bounds__(THREADS, ROWS > 1 ? 7 : 1024 / THREADS) balance_rows_kernel(const void* __restrict__ logits, int nq, int nlist, float a, const uint8_t* __restrict__ valid,
                                                               const int32_t* __restrict__ counts, int how_least, BalanceTotals* __restrict__ totals,
                                                               uint32_t* __restrict__ ticket, float4* __restrict__ stats, float* __restrict__ loss) {
    using P = LogitPiece<BF16>;
    __shared__ BalanceSums part[THREADS / 32][ROWS];
    __shared__ float4 mine[ROWS];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int q0 = blockIdx.x * ROWS, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t T = totals->slots;
    int base = 0;
    if (how_least == BALANCE_LEAST_KEPT) base = balance_kept(totals);
    BalanceSums S[ROWS];
    bool counted[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        S[r] = balance_none(a);
        counted[r] = q0 + r < nq && (!valid || valid[q0 + r]);
    }
    if (ROWS == 1) {
        if (how_least == BALANCE_LEAST_OWN) base = balance_least<THREADS>(counts, nlist);
        if (counted[0]) balance_sweep<BF16>(S[0], logits, (size_t)q0 * nlist, nlist, a, counts, base, tid, THREADS);
    } else if (!WHOLE) {
        if (how_least == BALANCE_LEAST_OWN) base = balance_least<THREADS>(counts, nlist);
        int head[ROWS], pieces[ROWS], most = 0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            head[r] = pieces[r] = 0;
            if (!counted[r]) continue;
            const size_t row = (size_t)(q0 + r) * nlist;
            head[r] = balance_head<BF16>(logits, row, nlist);
            pieces[r] = (nlist - head[r]) / P::UNIT;
            most = max(most, pieces[r]);
            const int tail = head[r] + pieces[r] * P::UNIT;
            for (int i = tid; i < head[r] + (nlist - tail); i += THREADS) {
                const int l = i < head[r] ? i : tail + (i - head[r]);
                const float v[1] = {load_l<BF16>(logits, row + l)}, c[1] = {(float)(counts[l] - base)};
                balance_add<1>(S[r], v, c, a);
            }
        }
        for (int p = tid; p < most; p += THREADS) {
            uint4 w[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (p < pieces[r]) w[r] = P::load(logits, (size_t)(q0 + r) * nlist + head[r] + (size_t)p * P::UNIT);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (p < pieces[r]) {
                    float c[P::UNIT], v[P::UNIT];
                    balance_window<BF16>(counts, head[r] + p * P::UNIT, nlist, base, c);
                    P::values(w[r], v);
                    balance_add<P::UNIT>(S[r], v, c, a);
                }
        }
    } else {
        uint4 next[ROWS];  // the piece behind is on its way while this one is added
        auto fetch = [&](int l) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (counted[r] && l < nlist) next[r] = P::load(logits, (size_t)(q0 + r) * nlist + l);
        };
        fetch(tid * P::UNIT);
        if (how_least == BALANCE_LEAST_OWN) base = balance_least<THREADS>(counts, nlist);
        for (int l = tid * P::UNIT; l < nlist; l += THREADS * P::UNIT) {
            uint4 w[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) w[r] = next[r];
            fetch(l + THREADS * P::UNIT);
            float c[P::UNIT];
            P::counts(counts, l, base, c);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (counted[r]) {
                    float v[P::UNIT];
                    P::values(w[r], v);
                    balance_add<P::UNIT>(S[r], v, c, a);
                }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        balance_join_warp(S[r], a);
        if (lane == 0) part[warp][r] = S[r];
    }
    __syncthreads();
    if (tid < ROWS) {
        BalanceSums s = part[0][tid];
        for (int w = 1; w < THREADS / 32; ++w) balance_join(s, part[w][tid], a);
        mine[tid] = balance_stats(s, T);
    }
    balance_close<ROWS, THREADS>(mine, q0, nq, nlist, T, base, totals, ticket, stats, loss);
}

// nq = 0: no row writes the loss
__global__ void balance_empty_kernel(BalanceTotals* __restrict__ totals, float* __restrict__ loss) {
    grid_dependency_wait();
    grid_dependents_may_launch();
    totals->per_row = totals->per_slot = 0.f;
    *loss = 0.f;
}

// ---- backward ----------------------------------------------------------------------------------------------------------------
struct BalanceBack { float k, per_slot; int base; };
__device__ __forceinline__ BalanceBack balance_back(const BalanceTotals* totals, const float* grad_loss, float scale) {
    return {grad_loss[0] * totals->per_row * scale, totals->per_slot, (int)totals->rows};
}
template <int n>
__device__ __forceinline__ void balance_grads(float (&v)[n], const float (&c)[n], float a, const BalanceBack& B, const float4& st) {
    const float m = B.k * st.y;
#pragma unroll
    for (int j = 0; j < n; ++j) v[j] = balance_exp2((v[j] - st.x) * a) * m * fmaf(c[j], B.per_slot, -st.z);
}

// Rows and counts of whole aligned pieces: a thread per piece of ROWS rows, which share the counts
template <bool BF16, int ROWS>
__global__ void __launch_bounds__(BALANCE_THREADS, 6) balance_backward_kernel(const void* __restrict__ logits, int nq, int nlist, float a, float scale,
                                                                           const uint8_t* __restrict__ valid, const int32_t* __restrict__ counts,
                                                                           const float4* __restrict__ stats, const BalanceTotals* __restrict__ totals,
                                                                           const float* __restrict__ grad_loss, void* __restrict__ out) {
    using P = LogitPiece<BF16>;
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int pieces = nlist / P::UNIT;
    const int64_t i = (int64_t)blockIdx.x * BALANCE_THREADS + threadIdx.x;
    const int q0 = (int)(i / pieces) * ROWS, l = (int)(i % pieces) * P::UNIT;
    if (q0 >= nq) return;
    uint4 w[ROWS];
    float c[P::UNIT];
    bool counted[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        counted[r] = q0 + r < nq && (!valid || valid[q0 + r]);
        if (counted[r]) w[r] = P::load(logits, (size_t)(q0 + r) * nlist + l);
    }
    const BalanceBack B = balance_back(totals, grad_loss, scale);
    P::counts(counts, l, B.base, c);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (q0 + r >= nq) break;
        float v[P::UNIT] = {};
        if (counted[r]) {
            P::values(w[r], v);
            balance_grads<P::UNIT>(v, c, a, B, stats[q0 + r]);
        }
        P::store(out, (size_t)(q0 + r) * nlist + l, v);
    }
}

// Long rows that start anywhere: a CTA takes BALANCE_THREADS pieces of BALANCE_ANY_ROWS rows one after the other (the counts are met again in L1).  Pieces
// follow the boundaries of the output; the logits, whose rows may start elsewhere, are read one at a time then.
constexpr int BALANCE_ANY_ROWS = 4;
template <bool BF16>
__global__ void __launch_bounds__(BALANCE_THREADS) balance_backward_long_kernel(const void* __restrict__ logits, int nq, int nlist, int spans, float a, float scale,
                                                                               const uint8_t* __restrict__ valid, const int32_t* __restrict__ counts,
                                                                               const float4* __restrict__ stats, const BalanceTotals* __restrict__ totals,
                                                                               const float* __restrict__ grad_loss, void* __restrict__ out) {
    using P = LogitPiece<BF16>;
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int span = blockIdx.x % spans, q0 = blockIdx.x / spans * BALANCE_ANY_ROWS, p = span * BALANCE_THREADS + threadIdx.x;
    const BalanceBack B = balance_back(totals, grad_loss, scale);
#pragma unroll
    for (int r = 0; r < BALANCE_ANY_ROWS; ++r) {
        const int q = q0 + r;
        if (q >= nq) break;
        const bool counted = !valid || valid[q];
        const size_t row = (size_t)q * nlist;
        const int head = balance_head<BF16>(out, row, nlist), pieces = (nlist - head) / P::UNIT, tail = head + pieces * P::UNIT;
        const float4 st = counted ? stats[q] : make_float4(0.f, 0.f, 0.f, 0.f);
        if (p < pieces) {
            const int l = head + p * P::UNIT;
            float v[P::UNIT] = {}, c[P::UNIT];
            if (counted) {
                if (((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0) {
                    P::values(P::load(logits, row + l), v);
                } else {
#pragma unroll
                    for (int i = 0; i < P::UNIT; ++i) v[i] = load_l<BF16>(logits, row + l + i);
                }
                balance_window<BF16>(counts, l, nlist, B.base, c);
                balance_grads<P::UNIT>(v, c, a, B, st);
            }
            P::store(out, row + l, v);
        }
        if (span == 0)
            for (int i = threadIdx.x; i < head + (nlist - tail); i += BALANCE_THREADS) {
                const int l = i < head ? i : tail + (i - head);
                float v[1] = {0.f}, c[1] = {(float)(counts[l] - B.base)};
                if (counted) {
                    v[0] = load_l<BF16>(logits, row + l);
                    balance_grads<1>(v, c, a, B, st);
                }
                if (BF16) static_cast<__nv_bfloat16*>(out)[row + l] = __float2bfloat16_rn(v[0]);
                else static_cast<float*>(out)[row + l] = v[0];
            }
    }
}

// Short rows that start anywhere: what lies in front of a row's first 16-byte boundary, its pieces and what lies behind the last are its slots; a CTA takes
// 2^tile_log2 slots of as many rows as its threads then make up, twice, so that the counts are met again in L1.  Pieces follow the
// boundaries of the output; logits whose rows start elsewhere are read one at a time.
template <bool BF16>
__global__ void __launch_bounds__(BALANCE_THREADS, 4) balance_backward_short_kernel(const void* __restrict__ logits, int nq, int nlist, int tiles, int tile_log2, float a,
                                                                                  float scale, const uint8_t* __restrict__ valid, const int32_t* __restrict__ counts,
                                                                                  const float4* __restrict__ stats, const BalanceTotals* __restrict__ totals,
                                                                                  const float* __restrict__ grad_loss, void* __restrict__ out) {
    using P = LogitPiece<BF16>;
    constexpr int TWICE = 2;
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int rows = BALANCE_THREADS >> tile_log2, slot = ((blockIdx.x % tiles) << tile_log2) + (threadIdx.x & ((1 << tile_log2) - 1));
    const int q0 = blockIdx.x / tiles * (rows * TWICE) + (threadIdx.x >> tile_log2);
    const bool alike = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    int begin[TWICE], n[TWICE];  // numbers of this slot
    bool counted[TWICE];
    uint4 w[TWICE];
    float4 st[TWICE];
#pragma unroll
    for (int r = 0; r < TWICE; ++r) {
        const int q = q0 + r * rows;
        begin[r] = n[r] = 0;
        counted[r] = false;
        if (q >= nq) continue;
        const size_t row = (size_t)q * nlist;
        const int head = balance_head<BF16>(out, row, nlist), pieces = (nlist - head) / P::UNIT;
        begin[r] = slot == 0 ? 0 : head + (slot - 1) * P::UNIT;
        n[r] = slot == 0 ? head : slot <= pieces ? P::UNIT : slot == pieces + 1 ? nlist - begin[r] : 0;
        counted[r] = !valid || valid[q];
        if (counted[r]) {
            st[r] = stats[q];
            if (n[r] == P::UNIT && alike) w[r] = P::load(logits, row + begin[r]);
        }
    }
    const BalanceBack B = balance_back(totals, grad_loss, scale);
#pragma unroll
    for (int r = 0; r < TWICE; ++r) {
        if (n[r] == 0) continue;
        const size_t at = (size_t)(q0 + r * rows) * nlist + begin[r];
        if (n[r] == P::UNIT) {
            float v[P::UNIT] = {}, c[P::UNIT];
            if (counted[r]) {
                if (alike) P::values(w[r], v);
                else {
#pragma unroll
                    for (int i = 0; i < P::UNIT; ++i) v[i] = load_l<BF16>(logits, at + i);
                }
                balance_window<BF16>(counts, begin[r], nlist, B.base, c);
                balance_grads<P::UNIT>(v, c, a, B, st[r]);
            }
            P::store(out, at, v);
        } else {
            for (int i = 0; i < n[r]; ++i) {
                float v[1] = {0.f}, c[1] = {(float)(counts[begin[r] + i] - B.base)};
                if (counted[r]) {
                    v[0] = load_l<BF16>(logits, at + i);
                    balance_grads<1>(v, c, a, B, st[r]);
                }
                if (BF16) static_cast<__nv_bfloat16*>(out)[at + i] = __float2bfloat16_rn(v[0]);
                else static_cast<float*>(out)[at + i] = v[0];
            }
        }
    }
}

// Rows and counts in whole, aligned pieces
static bool balance_whole(rago_dtype dtype, int nlist, const void* logits, const void* counts, const void* out) {
    return nlist % (dtype == RAGO_BF16 ? 8 : 4) == 0 &&
           (reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(counts) | reinterpret_cast<uintptr_t>(out)) % 16 == 0;
}

static rago_status balance_fail(rago_status st, const char* what, long long v = 0) {
    set_error(what, v);
    return st;
}

static rago_status balance_check(const void* logits, rago_dtype dtype, int32_t nq, int32_t nlist, float scale, float* a) {
    if (nq < 0) return balance_fail(RAGO_EINVAL, "nq = %lld is negative", nq);
    if (nlist < 1) return balance_fail(RAGO_EINVAL, "nlist = %lld must be at least 1", nlist);
    if (dtype != RAGO_F32 && dtype != RAGO_BF16) return balance_fail(RAGO_EINVAL, "dtype = %lld is neither F32 nor BF16", dtype);
    *a = (float)((double)scale * 1.44269504088896340736);
    if (!(scale - scale == 0.f) || scale == 0.f || !(*a - *a == 0.f) || *a == 0.f)
        return balance_fail(RAGO_EINVAL, "scale must be finite and not 0");
    // a difference of logits that leaves fp32 is a weight of 0 for every larger scale (units of their own for logits, as the policy's
    // scores have, took 4096 x 65 536 from 328 to 337 us)
    if (fabsf(scale) < 1e-36f) return balance_fail(RAGO_EUNSUPPORTED, "scale is below 1e-36 in magnitude");
    if (nq > 0 && !logits) return balance_fail(RAGO_EINVAL, "logits are null");
    if ((long long)nq * nlist >= (1LL << 40)) return balance_fail(RAGO_EUNSUPPORTED, "nq * nlist = %lld is 2^40 or more", (long long)nq * nlist);
    if (reinterpret_cast<uintptr_t>(logits) % (dtype == RAGO_F32 ? 4 : 2)) return balance_fail(RAGO_EALIGN, "logits are not aligned to their type");
    return RAGO_OK;
}

static rago_status balance_done(cudaError_t e, int launches, const char* what) {
    count_launch(launches);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return RAGO_OK;
    set_error("%s: %s", what, cudaGetErrorString(e));
    return RAGO_ECUDA;
}

}  // namespace rago

using namespace rago;

extern "C" rago_status rago_list_balance(const void* logits, rago_dtype dtype, int32_t nq, int32_t nlist, float scale, const int32_t* lists,
                                         int32_t nprobe, const uint8_t* valid, float* out_loss, int32_t* out_counts, float* out_stats,
                                         void* cuda_stream) {
    float a;
    const rago_status st = balance_check(logits, dtype, nq, nlist, scale, &a);
    if (st != RAGO_OK) return st;
    if (nprobe < 1) return balance_fail(RAGO_EINVAL, "nprobe = %lld must be at least 1", nprobe);
    if ((long long)nq * nprobe >= (1LL << 31)) return balance_fail(RAGO_EUNSUPPORTED, "nq * nprobe = %lld exceeds 2^31 - 1", (long long)nq * nprobe);
    if ((nq > 0 && !lists) || !out_loss || !out_counts || !out_stats) return balance_fail(RAGO_EINVAL, "null pointer");
    if (reinterpret_cast<uintptr_t>(out_stats) % 16) return balance_fail(RAGO_EALIGN, "out_stats need 16-byte alignment");
    if ((reinterpret_cast<uintptr_t>(lists) | reinterpret_cast<uintptr_t>(out_loss) | reinterpret_cast<uintptr_t>(out_counts)) % 4)
        return balance_fail(RAGO_EALIGN, "lists, out_loss or out_counts are not aligned to their type");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    float4* stats = reinterpret_cast<float4*>(out_stats);
    BalanceTotals* totals = reinterpret_cast<BalanceTotals*>(stats + nq);
    uint32_t* ticket = reinterpret_cast<uint32_t*>(totals);  // the first word
    const int64_t slots = (int64_t)nq * nprobe;
    int ranges = (int)parts_of(nlist, BALANCE_RANGE_LISTS), launches = 0;
    ranges = ranges < BALANCE_RANGE_CTAS ? ranges : BALANCE_RANGE_CTAS;
    const int range = (int)parts_of(nlist, ranges);
    cudaError_t e;
    const bool ranges_do = slots <= BALANCE_RANGE_SLOTS && range <= BALANCE_SHARED_LISTS;
    const int how_least = slots < nlist ? BALANCE_LEAST_0 : ranges_do || nlist <= BALANCE_OWN_LEAST ? BALANCE_LEAST_OWN : BALANCE_LEAST_KEPT;
    if (ranges_do) {
        e = launch_overlapped(balance_count_ranges_kernel, dim3((unsigned)parts_of(nlist, range)), dim3(BALANCE_RANGE_THREADS), (size_t)range * 4, s, lists, valid,
                              nq, nprobe, nlist, range, out_counts, totals, ticket);
        ++launches;
    } else {
        const bool shared = nlist <= BALANCE_SHARED_LISTS;
        e = launch_overlapped(balance_clear_kernel, dim3((unsigned)parts_of(nlist, BALANCE_THREADS)), dim3(BALANCE_THREADS), 0, s,
                              out_counts, nlist, totals, ticket);
        ++launches;
        if (e == cudaSuccess && slots) {
            const int64_t ctas = parts_of(slots, 8 * BALANCE_COUNT_THREADS);
            e = launch_overlapped(shared ? balance_count_kernel<true> : balance_count_kernel<false>, dim3((unsigned)(ctas < 4096 ? ctas : 4096)), dim3(BALANCE_COUNT_THREADS),
                                  shared ? (size_t)nlist * 4 : 0, s, lists, valid, nq, nprobe, nlist, how_least == BALANCE_LEAST_KEPT, out_counts, totals);
            ++launches;
        }
    }
    if (e == cudaSuccess) {
        ++launches;
        const bool whole = balance_whole(dtype, nlist, logits, out_counts, nullptr);
        auto rows = [&](auto bf16) {
            constexpr bool B = decltype(bf16)::value;
            auto launch = [&](auto kernel, int per_cta, int threads) {
                return launch_overlapped(kernel, dim3((unsigned)parts_of(nq, per_cta)), dim3((unsigned)threads), 0, s, logits, nq, nlist, a, valid, out_counts, how_least,
                                         totals, ticket, stats, out_loss);
            };
            auto launch_short = [&](auto kernel, int per_cta) {
                return launch_overlapped(kernel, dim3((unsigned)parts_of(nq, per_cta)), dim3(BALANCE_THREADS), 0, s, logits, nq, nlist, a, valid, out_counts, totals, ticket,
                                         stats, out_loss);
            };
            // What a row is given, each rule with the forward pass's us on its two sides (in a stream of such passes, rows x lists, fp32 unless bf16 is said):
            // up to 16 pieces 8 lanes: 16 384 x 64 10.8, a warp 16.8; 16 384 x 128 bf16 11.7 and 19.1
            if (nlist <= (B ? 128 : 64)) return launch_short(balance_short_rows_kernel<B, 8, 1>, 32);
            // up to 1024 lists a warp: 1000 x 512 9.3, a CTA 10.7; 8192 x 1024 21.4 and 23.5, but 1000 x 1024 12.0 and 10.4, 8192 x 2048 31.6 and
            // 29.1 (64 rows would take a CTA each from 512 lists on: 9.2 and 6.5); two rows a warp from 8192 rows: 8192 x 512 16.6, one 19.2, but
            // 4096 x 512 13.6 and 11.9
            if (nlist <= BALANCE_SHORT_LISTS) return nq >= 8192 ? launch_short(balance_short_rows_kernel<B, 32, 2>, 16) : launch_short(balance_short_rows_kernel<B, 32, 1>, 8);
            // four rows a CTA of 128 threads where that fills the GPU: 16 384 x 4096 bf16 56, two 63; 4096 x 65 536 185 and 210 (in bf16 129 and 123), but
            // 2048 x 65 536 bf16 94 and 73, 2048 x 4095 23.3 and 18.2
            if (nq >= 4096) return whole ? launch(balance_rows_kernel<B, 4, true, 128>, 4, 128) : launch(balance_rows_kernel<B, 4, false, 128>, 4, 128);
            // two: 1024 x 65 536 bf16 51.5, one 54.0; 2048 x 4096 15.5 and 22.2
            if (nq >= 1024) return whole ? launch(balance_rows_kernel<B, 2, true, 128>, 2, 128) : launch(balance_rows_kernel<B, 2, false, 128>, 2, 128);
            // one: 600 x 8192 17.6, with 256 threads 18.7; fewer rows with 256: 300 x 4096 8.6, with 128 10.8, with 512 11.0; longer ones with 512:
            // 128 x 32 768 bf16 11.4, with 256 15.6
            if (nq >= 512) return launch(balance_rows_kernel<B, 1, false, 128>, 1, 128);
            return nlist >= 16384 ? launch(balance_rows_kernel<B, 1, false, 512>, 1, 512) : launch(balance_rows_kernel<B, 1, false, 256>, 1, 256);
        };
        if (nq == 0) e = launch_overlapped(balance_empty_kernel, dim3(1), dim3(1), 0, s, totals, out_loss);
        else e = dtype == RAGO_BF16 ? rows(std::true_type{}) : rows(std::false_type{});
    }
    return balance_done(e, launches, "list balance kernels");
}

extern "C" rago_status rago_list_balance_backward(const void* logits, rago_dtype dtype, int32_t nq, int32_t nlist, float scale, const uint8_t* valid,
                                                  const int32_t* counts, const float* stats, const float* grad_loss, void* grad_logits,
                                                  void* cuda_stream) {
    float a;
    const rago_status st = balance_check(logits, dtype, nq, nlist, scale, &a);
    if (st != RAGO_OK || nq == 0) return st;
    if (!counts || !stats || !grad_loss || !grad_logits) return balance_fail(RAGO_EINVAL, "null pointer");
    if (reinterpret_cast<uintptr_t>(stats) % 16) return balance_fail(RAGO_EALIGN, "stats need 16-byte alignment");
    if ((reinterpret_cast<uintptr_t>(counts) | reinterpret_cast<uintptr_t>(grad_loss)) % 4) return balance_fail(RAGO_EALIGN, "counts or grad_loss are not aligned to their type");
    if (reinterpret_cast<uintptr_t>(grad_logits) % (dtype == RAGO_F32 ? 4 : 2)) return balance_fail(RAGO_EALIGN, "grad_logits are not aligned to their type");
    const float4* st4 = reinterpret_cast<const float4*>(stats);
    const BalanceTotals* totals = reinterpret_cast<const BalanceTotals*>(st4 + nq);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool whole = balance_whole(dtype, nlist, logits, counts, grad_logits);
    auto go = [&](auto bf16) {
        constexpr bool B = decltype(bf16)::value;
        const int64_t pieces = nlist / (B ? 8 : 4), per = BALANCE_THREADS;
        if (!whole) {
            if (pieces >= per) {  // 4096 x 65 533 in bf16: 260 us, by slots 334 (267 now); 16 384 x 61: 17.6, by slots 5.2
                const int spans = (int)parts_of(pieces, per);
                return launch_overlapped(balance_backward_long_kernel<B>, dim3((unsigned)(spans * parts_of(nq, BALANCE_ANY_ROWS))),
                                         dim3(BALANCE_THREADS), 0, s, logits, nq, nlist, spans, a, scale, valid, counts, st4, totals, grad_loss, grad_logits);
            }
            const int64_t slots = pieces + 2;
            int tile_log2 = 1;
            while (tile_log2 < 8 && (1 << tile_log2) < slots) ++tile_log2;
            const int tiles = (int)((slots + (1 << tile_log2) - 1) >> tile_log2), rows = 2 * (BALANCE_THREADS >> tile_log2);
            return launch_overlapped(balance_backward_short_kernel<B>, dim3((unsigned)(tiles * parts_of(nq, rows))), dim3(BALANCE_THREADS), 0, s, logits,
                                     nq, nlist, tiles, tile_log2, a, scale, valid, counts, st4, totals, grad_loss, grad_logits);
        }
        auto launch = [&](auto kernel, int64_t ctas) {
            return launch_overlapped(kernel, dim3((unsigned)ctas), dim3(BALANCE_THREADS), 0, s, logits, nq, nlist, a, scale, valid, counts, st4, totals, grad_loss,
                                     grad_logits);
        };
        if ((int64_t)nq * pieces >= (1 << 20)) return launch(balance_backward_kernel<B, 4>, parts_of(parts_of(nq, 4) * pieces, per));
        return launch(balance_backward_kernel<B, 1>, parts_of(nq * pieces, per));
    };
    return balance_done(dtype == RAGO_BF16 ? go(std::true_type{}) : go(std::false_type{}), 1, "list balance backward kernel");
}
