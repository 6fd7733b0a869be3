// Rows in 4 bits with group scales: scores of a whole store, re-scoring of candidates, gradient to the queries.
//
// row n, number i = s[n][i / group] * (c - 8), c = nibble i of the row, low nibble first.  All sums are fp32; the scale of a
// group is taken out of the sum over it, so a product is rounded as fp32 rounds it and nothing else is.
#include <atomic>
#include <type_traits>

#include <cuda_fp16.h>

#include "common.cuh"

namespace rago {

constexpr int Q4_MAX_D = 8192;

struct Q4Rows {
    const uint8_t* codes;
    const void* scales;
    int64_t N;
    int d, group, groups;  // groups = ceil(d / group)
};

template <bool BF16>
__device__ __forceinline__ float load_f(const void* base, size_t i) {
    if (BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[i]);
    return static_cast<const float*>(base)[i];
}
// ---- scores of every row -----------------------------------------------------------------------------------------------
// 2 nq N d operations on N d / 2 bytes: for few queries the rows' bytes bound it, so the work per byte has to be small.  A small number
// put into the mantissa of a power of two that is then taken off is a published way around conversions (Kim, Henry, Fahim and Hassan
// Awadalla, "Who Says Elephants Can't Run", 2022, for 4 and 8 bits and fp16); here c - 8, exact in fp16, costs 1.1 instructions a number:
// nibbles i and i + 4 of a word are masked into the mantissas of two 1024s at a time (16 c in place of c for every second pair, which
// saves the shift), one fp16 instruction takes the rest off.  The matrix instruction (m16n8k16, 16 rows by 8 queries, fp32 sums) does
// the products.
// Queries go in as fp16 after a power of two per query that brings its largest number to 2^14 .. 2^15 (taken off the sums again):
// a bf16 number fits as it is, an fp32 number is cut into two parts, hi = fp16(x) and fp16(x - hi), 23 of its 24 bits: off by at
// most 2^-23 of itself, or by 2^-39 of the query's largest number where that is more.  (A third part for the last bit would be half as many
// matrix instructions again; that bit lies below the rounding of the fp32 sums: 7e-8 of the scores' size against 64 bits, plain fp32
// sums 1.3e-7.)  The parts'
// products add up in the same fp32 accumulators; up to four fp32 queries put their parts side by side into the eight columns, so that
// one instruction does for all of them.  The sum over a group is multiplied by the row's scale and added to the row's total.
//
// A warp owns 32 rows at a time and runs on its own: it keeps a ring of copies (cp.async, 64 bytes of each row a stage) going
// across its tiles and never meets the other warps of its CTA, which share the queries in shared memory only.  The order of a row's
// numbers is permuted alike in rows and queries: thread t of a quad takes word t of every 16 bytes, whatever the group.
//
// Measured: 10 M rows of 1024 (groups of 128) for 8 bf16 queries 985 to 1 050 us in twenty calls at 1 965 MHz (5.3 to 5.7 TB/s), 1 170 to 1 240 in
// a stream of thousands, where 1 kW holds the clock at 1 640 to 1 560 MHz; bound by unpacking (2.4 instructions a number and lane, 70% of
// the issue slots).  100 000 rows of 768 for one fp32 query 15 us, 4 of them before the first product; 1 000 003 rows of 768 (groups of 32)
// for 37 queries 228 us, where each group's 80 sums a lane are scaled between the matrix instructions.
constexpr int Q4S_ROWS = 32, Q4S_STRIDE = 80;  // 64 bytes of a row a stage, spaced 20 words: the 8 rows of a fragment meet no bank twice
constexpr int Q4S_STAGE = Q4S_ROWS * Q4S_STRIDE;
// Most tiles of columns (times parts) for which warps may share a tile of rows.  (1000 rows of 768 for one query 4.1 us, not shared 4.9; three and four
// tiles gain less, 1000 rows for 20 bf16 queries 6.2 instead of 7.3 and nothing at 100 000, for as many kernels more.)  Kernels of 8
// warps are built for as many tiles, and the plan asks for them with up to two.
constexpr int Q4S_SPLIT_TILES = 2;
constexpr int Q4S_MAX_TILES = 8, Q4S_MAX_NQ = 8 * Q4S_MAX_TILES;  // eight queries a tile

enum { Q4_BF16 = 0, Q4_F32 = 1, Q4_F32_PACKED = 2 };  // how queries go in; parts side by side in the tiles' order: 1, 2, 1

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// An instruction takes one constant; a second one has to sit in a register, and the compiler, which knows it, would rather load
// it again each time (3.2 instructions a number and lane instead of 2.7).  These come out of something that it cannot know.
struct Q4Consts { uint32_t bias, less; };  // 1024 in both halves, -72 in both halves
__device__ __forceinline__ Q4Consts q4_consts(int nq) {
    const uint32_t zero = (uint32_t)nq >> 31;  // nq > 0
    return {0x64006400u + zero, 0xD480D480u + zero};
}
// The numbers of a word less 8, as pairs (i, i + 4) of fp16
__device__ __forceinline__ void q4_pairs(uint32_t word, const Q4Consts& K, uint32_t (&v)[4]) {
    const uint32_t high = word >> 8;
    auto biased = [&](uint32_t w, uint32_t mask) {
        uint32_t r;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(K.bias));  // (w & mask) | bias
        return r;
    };
    auto low_pair = [&](uint32_t w) {  // 1024 + c
        const uint32_t b = biased(w, 0x000F000Fu);
        const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&b), __half2half2(__ushort_as_half(0x6408)));
        return *reinterpret_cast<const uint32_t*>(&r);
    };
    auto high_pair = [&](uint32_t w) {  // 1024 + 16 c
        const uint32_t b = biased(w, 0x00F000F0u);
        const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&b), __half2half2(__ushort_as_half(0x2C00)), *reinterpret_cast<const __half2*>(&K.less));
        return *reinterpret_cast<const uint32_t*>(&r);
    };
    v[0] = low_pair(word); v[1] = high_pair(word); v[2] = low_pair(high); v[3] = high_pair(high);
}

// Powers of two that bring the queries' largest numbers to 2^14 .. 2^15, and their reciprocals; 1 for a query that is zero; 1 and infinity
// for one that is not finite, whose results are all infinite or NaN.  A warp per query.
template <bool QBF16>
__device__ __forceinline__ void q4_query_units(float* __restrict__ unit, float* __restrict__ back, const void* __restrict__ queries, int q0, int nq, int d) {
    for (int q = threadIdx.x >> 5; q < nq; q += blockDim.x >> 5) {
        uint32_t top = 0;  // of the magnitudes' bits, which are ordered as the magnitudes are
        const size_t at = (size_t)(q0 + q) * d;
        for (int i = (threadIdx.x & 31) * 8; i < d; i += 256) {
            if (QBF16) {
                const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(queries) + at + i);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) top = max(top, max(w[j] & 0x7FFF0000u, (w[j] << 16) & 0x7FFF0000u));
            } else {
                const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(queries) + at + i);
#pragma unroll
                for (int j = 0; j < 2; ++j) top = max(top, max(max(p[j].x & 0x7FFFFFFFu, p[j].y & 0x7FFFFFFFu), max(p[j].z & 0x7FFFFFFFu, p[j].w & 0x7FFFFFFFu)));
            }
        }
        top = __reduce_max_sync(0xffffffffu, top);
        const int e = (int)(top >> 23);  // biased exponent
        int k = top == 0 || e == 255 ? 0 : 141 - e;
        k = k > 126 ? 126 : k;
        if ((threadIdx.x & 31) == 0) {
            unit[q] = __uint_as_float((uint32_t)(127 + k) << 23);
            back[q] = e == 255 ? __int_as_float(0x7f800000) : __uint_as_float((uint32_t)(127 - k) << 23);
        }
    }
}

// The queries in the order of the matrix fragments: block of 32 numbers, tile of 8 columns, part, lane -> 16 bytes, the pairs
// (i, i + 4), i = 0 .. 3, of the lane's word.  Zero behind d and behind nq.
template <int MODE>
__device__ __forceinline__ void q4_stage_queries(uint4* __restrict__ dst, const float* __restrict__ unit, const void* __restrict__ queries, int q0, int nq,
                                                 int d, int blocks, int tiles) {
    constexpr int PARTS = MODE == Q4_F32 ? 2 : 1;
    for (int u = threadIdx.x; u < blocks * tiles * 32; u += blockDim.x) {
        const int lane = u & 31, bt = u >> 5, tile = bt % tiles, i0 = bt / tiles * 32 + (lane & 3) * 8;
        const int col = lane >> 2, q = MODE == Q4_F32_PACKED ? (col & 3) : tile * 8 + col;
        float x[8] = {};
        if (q < nq && i0 < d) {
            const size_t at = (size_t)(q0 + q) * d + i0;
            if (MODE == Q4_BF16) {
                const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(queries) + at);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
            } else {
                const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(queries) + at);
                *reinterpret_cast<float4*>(x) = p[0];
                *reinterpret_cast<float4*>(x + 4) = p[1];
            }
            const float m = unit[q];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= m;
        }
        uint32_t h[PARTS][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __half hi = __float2half_rn(x[i]);
            const __half lo = __float2half_rn(x[i] - __half2float(hi));
            if (MODE == Q4_F32_PACKED) {
                h[0][i] = __half_as_ushort(col < 4 ? hi : lo);
            } else {
                h[0][i] = __half_as_ushort(hi);
                if (PARTS == 2) h[PARTS - 1][i] = __half_as_ushort(lo);
            }
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
            dst[(size_t)(bt * PARTS + p) * 32 + lane] = make_uint4(h[p][0] | h[p][4] << 16, h[p][1] | h[p][5] << 16, h[p][2] | h[p][6] << 16, h[p][3] | h[p][7] << 16);
    }
}

__device__ __forceinline__ uint32_t q4_lds(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint4 q4_lds4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}

// <query, row> as it stands, by one thread: the sum over a group, then its scale.  `x` is the query, fp32 or bf16.
template <bool QBF16, bool SBF16>
__device__ __forceinline__ float q4_score_direct(const uint8_t* __restrict__ codes, const void* __restrict__ scales, const void* __restrict__ x, int d, int group) {
    float total = 0.f;
    for (int i0 = 0; i0 < d; i0 += group) {
        float sum = 0.f;
        const int i1 = min(d, i0 + group);
        for (int i = i0; i < i1; ++i) sum = fmaf(load_f<QBF16>(x, i), (float)((codes[i >> 1] >> (4 * (i & 1))) & 15) - 8.f, sum);
        total = fmaf(load_f<SBF16>(scales, i0 / group), sum, total);
    }
    return total;
}

// The unit comes off last, so a total may leave the range of fp32 where the score, up to 2^140 times smaller, does not (a short query,
// large scales).  A warp that has met one looks the results of its tiles through and takes what is not finite again without a unit, number by
// number: rare, and right for all that fp32 holds.  A function of its own, called behind the last tile, and the rows' description left
// in the kernel's parameters: inlined, or with a copy of them on the stack, it cost the loop 3 to 8% (registers).
template <int MODE, bool SBF16, int NT>
__device__ __noinline__ void q4_scores_again(const Q4Rows& R, const void* __restrict__ queries, int q0, int nq, int split, const float* back, float* __restrict__ out) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, teams = (blockDim.x >> 5) / split;
    const int tiles = (int)((R.N + Q4S_ROWS - 1) / Q4S_ROWS), step = gridDim.x * teams;
    constexpr bool QB = MODE == Q4_BF16;
    for (int tile = warp / split * gridDim.x + blockIdx.x; tile < tiles; tile += step) {
        const int64_t last = R.N > Q4S_ROWS ? R.N - Q4S_ROWS : 0, top = (int64_t)tile * Q4S_ROWS < last ? (int64_t)tile * Q4S_ROWS : last;
#pragma unroll 1
        for (int i = 0; i < NT * 8; ++i) {
            const int q = (i >> 3) * 8 + 2 * t + (i & 1), r = g + 8 * ((i >> 1) & 3);
            if (q >= nq || (MODE == Q4_F32_PACKED && t >= 2) || r >= R.N || !(back[q] < __int_as_float(0x7f800000))) continue;
            float* const at = out + (size_t)(q0 + q) * R.N + top + r;
            if (fabsf(*at) < __int_as_float(0x7f800000)) continue;
            *at = q4_score_direct<QB, SBF16>(R.codes + (size_t)(top + r) * (R.d / 2), static_cast<const uint8_t*>(R.scales) + (size_t)(top + r) * R.groups * (SBF16 ? 2 : 4),
                                             static_cast<const uint8_t*>(queries) + (size_t)(q0 + q) * R.d * (QB ? 2 : 4), R.d, R.group);
        }
    }
}

// SBF16: scales in bf16; GB = group / 32; NT tiles of 8 queries; STAGES of a warp's ring.  `split` warps share the chunks of a tile
// (1 unless there are few rows): each sums its own part, the first adds the others' up.
template <int MODE, bool SBF16, int GB, int NT, int WARPS, int STAGES, bool SPLIT>
__global__ void __launch_bounds__(WARPS * 32, WARPS == 8 ? 2 : 1) q4_scores_kernel(const __grid_constant__ Q4Rows R, const void* __restrict__ queries, int q0, int nq, int shared_by,
                                                               float* __restrict__ out) {
    const int split = SPLIT ? shared_by : 1;
    constexpr int PARTS = MODE == Q4_F32 ? 2 : 1, ES = SBF16 ? 2 : 4;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float unit[Q4S_MAX_NQ], back[Q4S_MAX_NQ];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int all_chunks = (R.d + 127) / 128, member = warp % split, team = warp / split, teams = WARPS / split;
    const int chunk0 = all_chunks * member / split, chunks = all_chunks * (member + 1) / split - chunk0;  // stages of a tile, at least one
    const int xs_at = WARPS * STAGES * Q4S_STAGE;
    const uint32_t xs = smem_u32(smem) + xs_at + lane * 16 + chunk0 * (4 * NT * PARTS * 512);
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int tiles = (int)((R.N + Q4S_ROWS - 1) / Q4S_ROWS), step = gridDim.x * teams;
    const int first = team * gridDim.x + blockIdx.x;  // few tiles go to different SMs
    const int row_bytes = R.d / 2;
    // A tile's rows: the last tile is moved back to end with row N - 1 (rows that it shares with the tile before get the same
    // value twice); with less than 32 rows in all, the last one stands in for those that are missing.
    const int64_t last_row = R.N > Q4S_ROWS ? R.N - Q4S_ROWS : 0;
    auto top_row = [&](int tile) { const int64_t r = (int64_t)tile * Q4S_ROWS; return r < last_row ? r : last_row; };
    int row_of[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) row_of[r] = g + 8 * r < R.N ? g + 8 * r : (int)R.N - 1;

    // Copies run ahead of the arithmetic.  csrc: this lane's 16 bytes of the tile's first row in the chunk to copy next; cnext: the same
    // of the tile behind; ctiles: tiles left to copy.
    const int mine = first < tiles ? (tiles - first + step - 1) / step : 0;
    int cleft = chunks, ctiles = mine;
    const uint32_t ring = smem_u32(smem) + warp * STAGES * Q4S_STAGE + g * Q4S_STRIDE;
    uint32_t cdst = ring + t * 16;
    const uint32_t cend = cdst + STAGES * Q4S_STAGE;
    const uint8_t* const clast = R.codes + (size_t)last_row * row_bytes + chunk0 * 64 + t * 16;
    const size_t tile_bytes = (size_t)step * Q4S_ROWS * row_bytes;
    const uint8_t* csrc = R.codes + (size_t)top_row(first) * row_bytes + chunk0 * 64 + t * 16;
    const uint8_t* cnext = csrc + tile_bytes < clast ? csrc + tile_bytes : clast;
    const bool short_chunk = (chunk0 + chunks - 1) * 64 + t * 16 >= row_bytes;  // this lane has nothing in the last chunk
    uint32_t crow[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) crow[r] = row_of[r] * row_bytes;
    auto copy = [&] {
        if (ctiles > 0 && !(short_chunk && cleft == 1)) {
#pragma unroll
            for (int r = 0; r < 4; ++r) cp_async16(cdst + 8 * r * Q4S_STRIDE, csrc + crow[r]);
        }
        cp_async_commit();
        csrc += 64;
        if (--cleft == 0) { cleft = chunks; --ctiles; csrc = cnext; cnext = cnext + tile_bytes < clast ? cnext + tile_bytes : clast; }
        cdst += Q4S_STAGE;
        if (cdst == cend) cdst -= STAGES * Q4S_STAGE;
    };
    // This lane's share of a stage's scales: rows g + 8 r, the group that block t of the stage lies in; fetched a stage ahead.
    const int row_scales = R.groups * ES;
    const uint8_t* const slast = static_cast<const uint8_t*>(R.scales) + (size_t)last_row * row_scales + (chunk0 * 4 + t) / GB * ES;
    const size_t tile_scales = (size_t)step * Q4S_ROWS * row_scales;
    const uint8_t* ssrc = static_cast<const uint8_t*>(R.scales) + (size_t)top_row(first) * row_scales + (chunk0 * 4 + t) / GB * ES;
    const uint8_t* snext = ssrc + tile_scales < slast ? ssrc + tile_scales : slast;
    int sleft = chunks, stiles = mine;
    const bool short_scales = ((chunk0 + chunks - 1) * 4 + t) / GB >= R.groups;
    uint32_t srow[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) srow[r] = row_of[r] * row_scales;
    float next_scale[4] = {};
    auto load_scales = [&] {
        if (stiles > 0 && !(short_scales && sleft == 1)) {
#pragma unroll
            for (int r = 0; r < 4; ++r) next_scale[r] = load_f<SBF16>(ssrc + srow[r], 0);
        }
        ssrc += 4 / GB * ES;
        if (--sleft == 0) { sleft = chunks; --stiles; ssrc = snext; snext = snext + tile_scales < slast ? snext + tile_scales : slast; }
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) copy();
    load_scales();
    q4_query_units<MODE == Q4_BF16>(unit, back, queries, q0, nq, R.d);
    __syncthreads();
    q4_stage_queries<MODE>(reinterpret_cast<uint4*>(smem + xs_at), unit, queries, q0, nq, R.d, all_chunks * 4, NT);
    __syncthreads();

    const Q4Consts K = q4_consts(nq);
    uint32_t slot = ring + t * 4;
    const uint32_t slot_end = slot + STAGES * Q4S_STAGE;
    float finite = 0.f;  // NaN once a total is not
    for (int tile = first; tile < tiles; tile += step) {
        float total[2][NT][4] = {};
        uint32_t x = xs;
        for (int chunk = 0; chunk < chunks; ++chunk) {
            float scale[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) scale[r] = next_scale[r];
            load_scales();
            cp_async_wait<STAGES - 2>();
            __syncwarp();
            copy();  // into the slot that every lane has left
            float part[2][NT][4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                if (b % GB == 0) {
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) part[m][n][i] = 0.f;
                }
                uint32_t a[2][2][4];  // row tile, half of the word, fragment
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t v[4];
                        q4_pairs(q4_lds(slot + (16 * m + 8 * h) * Q4S_STRIDE + 16 * b), K, v);
                        a[m][0][h] = v[0];
                        a[m][0][h + 2] = v[1];
                        a[m][1][h] = v[2];
                        a[m][1][h + 2] = v[3];
                    }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) {
                        const uint4 v = q4_lds4(x + ((b * NT + n) * PARTS + p) * 512);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            mma_f16(part[m][n], a[m][0], v.x, v.y);
                            mma_f16(part[m][n], a[m][1], v.z, v.w);
                        }
                    }
                if (b % GB == GB - 1) {
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const int from = (lane & ~3) | (b - b % GB);
                        const float s0 = GB == 4 ? scale[2 * m] : __shfl_sync(0xffffffffu, scale[2 * m], from);
                        const float s1 = GB == 4 ? scale[2 * m + 1] : __shfl_sync(0xffffffffu, scale[2 * m + 1], from);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            total[m][n][0] = fmaf(s0, part[m][n][0], total[m][n][0]);
                            total[m][n][1] = fmaf(s0, part[m][n][1], total[m][n][1]);
                            total[m][n][2] = fmaf(s1, part[m][n][2], total[m][n][2]);
                            total[m][n][3] = fmaf(s1, part[m][n][3], total[m][n][3]);
                        }
                    }
                }
            }
            x += 4 * NT * PARTS * 512;
            slot += Q4S_STAGE;
            if (slot == slot_end) slot -= STAGES * Q4S_STAGE;
        }
        if (SPLIT) {  // the others' sums, in their order
            float* shared = reinterpret_cast<float*>(smem + xs_at + all_chunks * (4 * NT * PARTS * 512)) + warp * (2 * NT * 4 * 32) + lane;
            float* const flat = &total[0][0][0];
            if (member) {
#pragma unroll
                for (int i = 0; i < 2 * NT * 4; ++i) shared[i * 32] = flat[i];
            }
            named_bar_sync(1 + team, split * 32);
            if (!member) {
                for (int o = 1; o < split; ++o)
#pragma unroll
                    for (int i = 0; i < 2 * NT * 4; ++i) flat[i] += shared[(o * 2 * NT * 4 + i) * 32];
            }
            named_bar_sync(1 + team, split * 32);
            if (member) continue;
        }
        const int64_t top = top_row(tile);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                int q = n * 8 + 2 * t + c;
                const bool writes = q < nq && !(MODE == Q4_F32_PACKED && t >= 2);
                if (!writes) q = 0;
                const float u = back[q];
                float* dst = out + (size_t)(q0 + q) * R.N + top;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v = total[r / 2][n][2 * (r & 1) + c];
                    // column 4 p + q holds part p: threads t and t + 2 hold the two parts of a query
                    if (MODE == Q4_F32_PACKED) v += __shfl_xor_sync(0xffffffffu, v, 2);
                    finite = fmaf(v, 0.f, finite);
                    if (writes && g + 8 * r < R.N) __stcs(dst + row_of[r], v * u);
                }
            }
    }
    cp_async_wait<0>();
    if (!(finite == 0.f) && member == 0) q4_scores_again<MODE, SBF16, NT>(R, queries, q0, nq, split, back, out);
}

// ---- candidates -----------------------------------------------------------------------------------------------------------
// Rows are gathered, d / 2 bytes each; what has to be kept small again is the work per byte, now in fp32: the direct form of the
// distance is a difference and a square per number.  Nibble i of half a word is masked into the mantissa of 2^23 where it lies (16^i c),
// and one fused multiply-add takes it to c - 8, exactly; all fp32 arithmetic goes in pairs (fma.rn.f32x2; one at a time it is a third
// more instructions).  Measured: 4096 queries' 100 candidates of 768 numbers 65 us (inner product) and 71 (distance) against 29 of their
// bytes; 55% of the issue slots, the rest waits for gathered rows.  20 candidates of one query: 2.2 us.
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ F2 f2u(uint32_t lo, uint32_t hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ void f2_get(const F2& a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ F2 f2_fma(const F2& a, const F2& b, const F2& c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// Held in registers throughout (see Q4Consts)
struct Q4Float {
    uint32_t bias;            // 2^23
    F2 unit[2], less[2];      // 16^-i and what comes off then, i = 0, 1 and 2, 3
};
__device__ __forceinline__ Q4Float q4_float(int some) {
    const uint32_t zero = (uint32_t)some >> 31;  // some >= 0
    Q4Float K;
    K.bias = 0x4B000000u + zero;
    K.unit[0] = f2(1.f, 1.f / 16); K.unit[1] = f2(1.f / 256, 1.f / 4096);
    K.less[0] = f2(-8388616.f, -524296.f); K.less[1] = f2(-32776.f, -2056.f);
    return K;
}
// numbers 0 .. 3 of the low half of w, less 8
__device__ __forceinline__ void q4_four(uint32_t w, const Q4Float& K, F2 (&v)[2]) {
    uint32_t n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(n[i]) : "r"(w), "r"(0xFu << (4 * i)), "r"(K.bias));  // (w & mask) | bias
    v[0] = f2_fma(f2u(n[0], n[1]), K.unit[0], K.less[0]);
    v[1] = f2_fma(f2u(n[2], n[3]), K.unit[1], K.less[1]);
}

// A query in shared memory: 32 numbers after 32, the 16-byte pieces of each spread over the banks by its place
__device__ __forceinline__ int q4_spread(int chunk, int piece) { return chunk * 32 + ((piece ^ (chunk & 7)) << 2); }
template <bool QBF16>
__device__ __forceinline__ void q4_stage_query(float* __restrict__ xs, const void* __restrict__ queries, size_t at, int d) {
    for (int i = threadIdx.x * 8; i < d; i += blockDim.x * 8) {
        float x[8];
        if (QBF16) {
            const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(queries) + at + i);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
        } else {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(queries) + at + i);
            *reinterpret_cast<float4*>(x) = p[0];
            *reinterpret_cast<float4*>(x + 4) = p[1];
        }
        *reinterpret_cast<float4*>(xs + q4_spread(i / 32, i % 32 / 4)) = *reinterpret_cast<const float4*>(x);
        *reinterpret_cast<float4*>(xs + q4_spread(i / 32, i % 32 / 4 + 1)) = *reinterpret_cast<const float4*>(x + 4);
    }
}

// Inner products are scaled by the 32: a query's numbers may be as large as 2^119 before that leaves fp32 where scaled products would not.
// (A query beyond that taken in as 2^-8 of itself cost all others 5 to 8%: 65.7 -> 71.1 us at 4096 x 100 of 768.)
// LANES lanes to a row, two rows each: a warp takes 64 / LANES candidates at a time, the CTAs of a query (blockIdx.y) and their warps
// in turn.  A lane's next 32 numbers of both rows are on their way while it works on these.
constexpr int Q4R_WARPS = 4;
template <bool QBF16, bool SBF16, bool L2, int LANES>
__global__ void __launch_bounds__(Q4R_WARPS * 32) q4_rescore_kernel(const Q4Rows R, const void* __restrict__ queries, const int64_t* __restrict__ ids, int k,
                                                                    float* __restrict__ out) {
    extern __shared__ __align__(16) uint8_t smem[];
    float* xs = reinterpret_cast<float*>(smem);
    constexpr int TEAMS = 32 / LANES, PER = 2 * TEAMS;
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int lane = threadIdx.x & 31, c0 = lane % LANES, team = lane / LANES;
    const int chunks = R.d / 32, row_bytes = R.d / 2, group_shift = R.group == 32 ? 0 : R.group == 64 ? 1 : 2;
    const size_t q = blockIdx.x;
    const Q4Float K = q4_float(k);
    int64_t j = (int64_t)(blockIdx.y * Q4R_WARPS + (threadIdx.x >> 5)) * PER + team * 2;
    const int step = gridDim.y * Q4R_WARPS * PER;
    auto id_at = [&](int64_t i) { return i < k ? ids[q * k + i] : (int64_t)-1; };
    int64_t id[2] = {id_at(j), id_at(j + 1)};
    q4_stage_query<QBF16>(xs, queries, q * R.d, R.d);
    __syncthreads();
    for (; j - team * 2 < k; j += step) {  // the same for a whole warp
        bool there[2];
        const uint8_t* row[2];
        size_t scale_at[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            there[r] = id[r] >= 0 && id[r] < R.N;
            row[r] = R.codes + (there[r] ? (size_t)id[r] * row_bytes : 0);
            scale_at[r] = there[r] ? (size_t)id[r] * R.groups : 0;
        }
        uint4 w[2] = {};
        float s[2] = {};
        auto fetch = [&](int c) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (there[r] && c < chunks) {
                    w[r] = *reinterpret_cast<const uint4*>(row[r] + c * 16);
                    s[r] = load_f<SBF16>(R.scales, scale_at[r] + (c >> group_shift));
                }
        };
        fetch(c0);
        const int64_t next[2] = {id_at(j + step), id_at(j + step + 1)};
        F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
        float total[2] = {};
        for (int c = c0; c < chunks; c += LANES) {
            const uint32_t now[2][4] = {{w[0].x, w[0].y, w[0].z, w[0].w}, {w[1].x, w[1].y, w[1].z, w[1].w}};
            const float scale[2] = {s[0], s[1]};
            fetch(c + LANES);
            if (!L2) sum[0] = sum[1] = f2(0.f, 0.f);
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(xs + q4_spread(c, p));
                const F2 x2[2] = {{x.x}, {x.y}};
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    F2 v[2];
                    q4_four(p & 1 ? now[r][p / 2] >> 16 : now[r][p / 2], K, v);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (L2) {
                            const F2 t = f2_fma(f2(-scale[r], -scale[r]), v[h], x2[h]);
                            sum[r] = f2_fma(t, t, sum[r]);
                        } else {
                            sum[r] = f2_fma(x2[h], v[h], sum[r]);
                        }
                }
            }
            if (!L2) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float lo, hi;
                    f2_get(sum[r], lo, hi);
                    total[r] = fmaf(scale[r], lo + hi, total[r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (L2) {
                float lo, hi;
                f2_get(sum[r], lo, hi);
                total[r] = lo + hi;
            }
            for (int o = LANES / 2; o; o >>= 1) total[r] += __shfl_xor_sync(0xffffffffu, total[r], o);
            if (c0 == 0 && j + r < k) out[q * k + j + r] = there[r] ? total[r] : L2 ? __int_as_float(0x7f800000) : __int_as_float(0xff800000);
            id[r] = next[r];
        }
    }
}

// ---- gradient to the queries -----------------------------------------------------------------------------------------------
// sum_j g_j row_j, or 2 sum_j g_j (query - row_j) for the distance, in that form: taken apart into 2 (query sum_j g_j - sum_j g_j row_j) it
// would cancel where candidates are near, 3e-5 of the gradient for queries 0.01 |query| away.  A thread owns 16 numbers, 8 bytes of a row; teams of
// d / 16 threads take the candidates in turn, their sums meet in shared memory, where the query lies too.  With few queries a cluster of CTAs shares the candidates
// of one, and adds its sums up through distributed shared memory.  Missing candidates are left out when ids and gradients are staged, so
// nothing of theirs is looked at.  Measured: 1024 queries' 100 candidates of 768 numbers 28 us (distance; 22 for inner products), which is latency: ids, rows, sums of the
// teams, one after the other, in a CTA that lives for 20 rows a team.
constexpr int Q4B_THREADS = 512, Q4B_STAGE = 512, Q4B_MAX_CLUSTER = 8;  // candidates staged at a time

template <bool QBF16, bool SBF16, bool L2>
__global__ void __launch_bounds__(Q4B_THREADS, 2) q4_rescore_backward_kernel(const Q4Rows R, const void* __restrict__ queries, const int64_t* __restrict__ ids, int k,
                                                                             const float* __restrict__ grad, int teams, int cluster_log2, void* __restrict__ out) {
    extern __shared__ __align__(16) uint8_t smem[];
    float* sums = reinterpret_cast<float*>(smem);  // [teams][d]
    __shared__ uint32_t rows[Q4B_STAGE];
    __shared__ float gs[Q4B_STAGE];
    __shared__ int found[Q4B_THREADS / 32];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, per_row = R.d / 16, team = tid / per_row, part = tid - team * per_row, row_bytes = R.d / 2;
    const int cluster = 1 << cluster_log2, rank = blockIdx.x & (cluster - 1);
    const size_t q = blockIdx.x >> cluster_log2;
    const int j0 = (int)(((int64_t)k * rank) >> cluster_log2), j1 = (int)(((int64_t)k * (rank + 1)) >> cluster_log2);
    const bool works = team < teams;
    const Q4Float K = q4_float(k);
    float* const xs = sums + teams * R.d;  // the query, for the distance
    if (L2) q4_stage_query<QBF16>(xs, queries, q * R.d, R.d);
    F2 acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = f2(0.f, 0.f);
    const int grp = part * 16 / R.group;
    for (int64_t base = j0; base < j1; base += Q4B_STAGE) {  // k may be the largest int
        const int n = (int)min((int64_t)Q4B_STAGE, j1 - base);
        __syncthreads();
        int have = 0;
        for (int i0 = 0; i0 < n; i0 += threads) {  // keep the candidates that are there, in their order
            const int i = i0 + tid;
            const int64_t id = i < n ? ids[q * k + base + i] : -1;
            const float g = i < n ? grad[q * k + base + i] : 0.f;
            const bool there = id >= 0 && id < R.N;
            const uint32_t mask = __ballot_sync(0xffffffffu, there);
            if (lane == 0) found[warp] = __popc(mask);
            __syncthreads();
            int at = have;
            for (int w = 0; w < (threads >> 5); ++w) {
                if (w < warp) at += found[w];
                have += found[w];
            }
            if (there) {
                at += __popc(mask & ((1u << lane) - 1u));
                rows[at] = (uint32_t)id;
                gs[at] = g;
            }
            __syncthreads();
        }
        if (works) {
            constexpr int AT_ONCE = L2 ? 2 : 4;  // rows whose numbers are asked for together (four of them with gradients and scales apart spill)
            for (int i = team; i < have; i += AT_ONCE * teams) {
                uint2 w[AT_ONCE];
                float f[AT_ONCE], g[AT_ONCE];  // scale, gradient; without L2 f is their product
#pragma unroll
                for (int a = 0; a < AT_ONCE; ++a) {
                    const int now = i + a * teams;
                    w[a] = make_uint2(0, 0);
                    f[a] = g[a] = 0.f;
                    if (now < have) {
                        const size_t row = rows[now];
                        w[a] = *reinterpret_cast<const uint2*>(R.codes + row * row_bytes + part * 8);
                        f[a] = load_f<SBF16>(R.scales, row * R.groups + grp);
                        g[a] = gs[now];
                    }
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    F2 x[2];
                    if (L2) {
                        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(xs + q4_spread(part / 2, part % 2 * 4 + p));
                        x[0] = {v.x}; x[1] = {v.y};
                    }
#pragma unroll
                    for (int a = 0; a < AT_ONCE; ++a) {
                        const uint32_t word = p / 2 ? w[a].y : w[a].x;
                        F2 v[2];
                        q4_four(p & 1 ? word >> 16 : word, K, v);
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (L2) acc[2 * p + h] = f2_fma(f2(g[a], g[a]), f2_fma(f2(-f[a], -f[a]), v[h], x[h]), acc[2 * p + h]);
                            else acc[2 * p + h] = f2_fma(f2(g[a] * f[a], g[a] * f[a]), v[h], acc[2 * p + h]);
                    }
                }
            }
        }
    }
    if (works) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<ulonglong2*>(sums + team * R.d + part * 16 + 4 * i) = make_ulonglong2(acc[2 * i].v, acc[2 * i + 1].v);
    }
    __syncthreads();
    // teams, then CTAs, in their order
    if (teams > 1)
        for (int i = tid; i < R.d; i += threads) {
            float v = sums[i];
            for (int t = 1; t < teams; ++t) v += sums[t * R.d + i];
            sums[i] = v;
        }
    if (cluster > 1) cluster_sync_all();
    else __syncthreads();
    auto over_cluster = [&](const float* at) {
        if (cluster == 1) return *at;
        float v = 0.f;
        for (int c = 0; c < cluster; ++c) v += __uint_as_float(lds_cluster_u32(mapa_shared(smem_u32(at), c)));
        return v;
    };
    const int i0 = (R.d * rank) >> cluster_log2, i1 = (R.d * (rank + 1)) >> cluster_log2;
    for (int i = i0 + tid; i < i1; i += threads) {
        const float v = over_cluster(sums + i) * (L2 ? 2.f : 1.f);
        if (QBF16) static_cast<__nv_bfloat16*>(out)[q * R.d + i] = __float2bfloat16_rn(v);
        else static_cast<float*>(out)[q * R.d + i] = v;
    }
    if (cluster > 1) cluster_sync_all();  // a CTA's sums stay until every other one has read them
}

// ---- argument checks and launches ---------------------------------------------------------------------------------------
static rago_status fail_q4(rago_status st, const char* what, long long v) {
    set_error(what, v);
    return st;
}

// Common checks; on success *R describes the rows.
static rago_status q4_check(const uint8_t* codes, const void* scales, rago_dtype scale_dtype, int64_t N, int32_t d, int32_t group,
                            const void* queries, rago_dtype query_dtype, int32_t nq, Q4Rows* R) {
    if (N < 0) return fail_q4(RAGO_EINVAL, "N = %lld is negative", N);
    if (nq < 0) return fail_q4(RAGO_EINVAL, "nq = %lld is negative", nq);
    if (d < 1) return fail_q4(RAGO_EINVAL, "d = %lld must be positive", d);
    if (scale_dtype != RAGO_F32 && scale_dtype != RAGO_BF16) return fail_q4(RAGO_EINVAL, "scale_dtype = %lld is neither F32 nor BF16", scale_dtype);
    if (query_dtype != RAGO_F32 && query_dtype != RAGO_BF16) return fail_q4(RAGO_EINVAL, "query_dtype = %lld is neither F32 nor BF16", query_dtype);
    if (group != 32 && group != 64 && group != 128) return fail_q4(RAGO_EUNSUPPORTED, "group = %lld is not 32, 64 or 128", group);
    if (d % 32 != 0 || d > Q4_MAX_D) return fail_q4(RAGO_EUNSUPPORTED, "d = %lld must be a multiple of 32, at most 8192", d);
    if (N >= (1LL << 31)) return fail_q4(RAGO_EUNSUPPORTED, "N = %lld needs more than 31-bit row numbers", N);
    if (nq > 0 && !queries) return fail_q4(RAGO_EINVAL, "queries are null", 0);
    if (N > 0 && (!codes || !scales)) return fail_q4(RAGO_EINVAL, "codes or scales are null", 0);
    if (reinterpret_cast<uintptr_t>(codes) % 16) return fail_q4(RAGO_EALIGN, "codes need 16-byte alignment", 0);
    if (reinterpret_cast<uintptr_t>(queries) % 16) return fail_q4(RAGO_EALIGN, "queries need 16-byte alignment", 0);
    if (reinterpret_cast<uintptr_t>(scales) % (scale_dtype == RAGO_F32 ? 4 : 2)) return fail_q4(RAGO_EALIGN, "scales are not aligned to their type", 0);
    R->codes = codes; R->scales = scales; R->N = N; R->d = d; R->group = group; R->groups = (d + group - 1) / group;
    return RAGO_OK;
}

static rago_status q4_check_lists(int32_t nq, const int64_t* ids, int32_t k, int32_t metric, const void* dists) {
    if (k < 1) return fail_q4(RAGO_EINVAL, "k = %lld must be at least 1", k);
    if (metric != RAGO_L2 && metric != RAGO_IP) return fail_q4(RAGO_EINVAL, "metric = %lld is neither L2 nor IP", metric);
    if ((long long)nq * k >= (1LL << 31)) return fail_q4(RAGO_EUNSUPPORTED, "nq * k = %lld exceeds 2^31 - 1", (long long)nq * k);
    if (nq > 0 && (!ids || !dists)) return fail_q4(RAGO_EINVAL, "null pointer", 0);
    if (reinterpret_cast<uintptr_t>(ids) % 8 || reinterpret_cast<uintptr_t>(dists) % 4) return fail_q4(RAGO_EALIGN, "ids or distances are not aligned to their type", 0);
    return RAGO_OK;
}

static rago_status q4_done(cudaError_t e, int launches, const char* what) {
    count_launch(launches);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return RAGO_OK;
    set_error("%s: %s", what, cudaGetErrorString(e));
    return RAGO_ECUDA;
}

static cudaError_t q4_sms(int* sms) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    return e == cudaSuccess ? cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) : e;
}
// f(bf16 queries, bf16 scales, L2) as constants
template <class F>
static cudaError_t q4_types(rago_dtype query, rago_dtype scale, int metric, F f) {
    std::true_type y;
    std::false_type n;
    auto m = [&](auto q, auto s) { return metric == RAGO_L2 ? f(q, s, y) : f(q, s, n); };
    auto sc = [&](auto q) { return scale == RAGO_BF16 ? m(q, y) : m(q, n); };
    return query == RAGO_BF16 ? sc(y) : sc(n);
}

// How a launch of the scores kernel goes: queries it takes, as tiles of 8 columns; warps of a CTA; warps that share a tile of rows.
// Few columns are bound by the rows' bytes, or by unpacking them: two CTAs of 8 warps on an SM with four stages each.  More
// columns take registers and shared memory, and the matrix instructions more of the time: one CTA of 12 warps, three stages.
struct Q4ScoresPlan { int mode, nq, tiles, warps, per_sm, split; size_t smem; };

constexpr int Q4_DEVICES = 64;
constexpr size_t Q4S_SMEM_ONE = 225 * 1024, Q4S_SMEM_TWO = 112 * 1024;  // shared memory of a CTA, alone on its SM or one of two
constexpr size_t q4s_ring(int warps, int stages) { return (size_t)warps * stages * Q4S_STAGE; }

static Q4ScoresPlan q4_scores_plan(const Q4Rows& R, bool bf16, int nq, int sms) {
    Q4ScoresPlan P;
    const int chunks = (R.d + 127) / 128;
    const size_t tile = (size_t)chunks * 128 * 8 * 2;  // eight columns of fp16
    const size_t room = Q4S_SMEM_ONE - q4s_ring(12, 3);  // at least one tile of the longest rows
    P.mode = bf16 ? Q4_BF16 : (nq <= 4 || 2 * tile > room ? Q4_F32_PACKED : Q4_F32);
    const int per_tile = P.mode == Q4_F32_PACKED ? 4 : 8, parts = P.mode == Q4_F32 ? 2 : 1;
    int most = P.mode == Q4_F32_PACKED ? 1 : (int)(room / (parts * tile));
    if (most > (bf16 ? Q4S_MAX_TILES : 4)) most = bf16 ? Q4S_MAX_TILES : 4;
    if (most == 7) most = 6;
    P.tiles = (int)min((int64_t)most, parts_of(nq, per_tile));
    if (P.tiles == 7) P.tiles = 8;  // not built
    P.nq = nq < P.tiles * per_tile ? nq : P.tiles * per_tile;
    const size_t x = tile * P.tiles * parts;
    static_assert(Q4S_SPLIT_TILES >= 2, "kernels of 8 warps are built up to there");
    const bool two = P.tiles * parts <= 2 && q4s_ring(8, 4) + x <= Q4S_SMEM_TWO;
    P.warps = two ? 8 : 12;
    P.per_sm = two ? 2 : 1;
    // Few tiles of rows: warps share a tile where that shortens the longest warp's work, counted in rounds of all warps, by a
    // tenth or more (100 000 rows are 3125 tiles for 2368 warps: two rounds, or three of halves).
    P.split = 1;
    const int64_t tiles = (R.N + Q4S_ROWS - 1) / Q4S_ROWS, all_warps = (int64_t)sms * P.per_sm * P.warps;
    const size_t sums = (size_t)P.warps * 2 * P.tiles * 4 * 32 * 4;
    P.smem = q4s_ring(P.warps, two ? 4 : 3) + x;
    if (P.tiles * parts <= Q4S_SPLIT_TILES && P.smem + sums <= (two ? Q4S_SMEM_TWO : Q4S_SMEM_ONE)) {
        auto rounds = [&](int split) { return (double)((tiles * split + all_warps - 1) / all_warps) / split; };
        for (int split = 2; split <= chunks && P.warps % split == 0; split *= 2)
            if (rounds(split) < 0.9 * rounds(P.split)) P.split = split;
        if (P.split > 1) P.smem += sums;
    }
    return P;
}

template <int MODE, bool SBF16, int GB, int NT, int WARPS, int STAGES, bool SPLIT>
static cudaError_t q4_scores_launch_one(const Q4ScoresPlan& P, const Q4Rows& R, const void* queries, int q0, int dev, int sms, float* out, cudaStream_t s) {
    auto kernel = q4_scores_kernel<MODE, SBF16, GB, NT, WARPS, STAGES, SPLIT>;
    static std::atomic<int> ready[Q4_DEVICES];  // once per device: room for the queries
    if (dev >= Q4_DEVICES || !ready[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Q4S_SMEM_ONE);
        if (e != cudaSuccess) return e;
        if (dev < Q4_DEVICES) ready[dev].store(1, std::memory_order_release);
    }
    const int64_t tiles = (R.N + Q4S_ROWS - 1) / Q4S_ROWS, most = (int64_t)sms * P.per_sm;
    return launch_overlapped(kernel, dim3((unsigned)(tiles < most ? tiles : most)), dim3(WARPS * 32), P.smem, s, R, queries, q0, P.nq, P.split, out);
}

template <int GB>
static cudaError_t q4_scores_launch(const Q4ScoresPlan& P, const Q4Rows& R, int scale_bf16, const void* queries, int q0, int dev, int sms, float* out, cudaStream_t s) {
    auto one = [&](auto mode, auto nt) {
        constexpr int MODE = decltype(mode)::value, NT = decltype(nt)::value;
        auto go = [&](auto warps, auto stages, auto shares) {
            constexpr int W = decltype(warps)::value, ST = decltype(stages)::value;
            constexpr bool SP = decltype(shares)::value;
            return scale_bf16 ? q4_scores_launch_one<MODE, true, GB, NT, W, ST, SP>(P, R, queries, q0, dev, sms, out, s)
                              : q4_scores_launch_one<MODE, false, GB, NT, W, ST, SP>(P, R, queries, q0, dev, sms, out, s);
        };
        using std::integral_constant;
        if constexpr (NT * (MODE == Q4_F32 ? 2 : 1) <= Q4S_SPLIT_TILES) {
            auto shares = [&](auto warps, auto stages) { return P.split > 1 ? go(warps, stages, std::true_type{}) : go(warps, stages, std::false_type{}); };
            if (P.warps == 8) return shares(integral_constant<int, 8>{}, integral_constant<int, 4>{});
            return shares(integral_constant<int, 12>{}, integral_constant<int, 3>{});
        } else {
            return go(integral_constant<int, 12>{}, integral_constant<int, 3>{}, std::false_type{});
        }
    };
    using std::integral_constant;
    if (P.mode == Q4_F32_PACKED) return one(integral_constant<int, Q4_F32_PACKED>{}, integral_constant<int, 1>{});
    if (P.mode == Q4_F32) {
        switch (P.tiles) {
            case 1: return one(integral_constant<int, Q4_F32>{}, integral_constant<int, 1>{});
            case 2: return one(integral_constant<int, Q4_F32>{}, integral_constant<int, 2>{});
            case 3: return one(integral_constant<int, Q4_F32>{}, integral_constant<int, 3>{});
            default: return one(integral_constant<int, Q4_F32>{}, integral_constant<int, 4>{});
        }
    }
    switch (P.tiles) {
        case 1: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 1>{});
        case 2: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 2>{});
        case 3: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 3>{});
        case 4: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 4>{});
        case 5: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 5>{});
        case 6: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 6>{});
        default: return one(integral_constant<int, Q4_BF16>{}, integral_constant<int, 8>{});
    }
}

}  // namespace rago

using namespace rago;

extern "C" rago_status rago_q4_scores(const uint8_t* codes, const void* scales, rago_dtype scale_dtype, int64_t N, int32_t d,
                                      int32_t group, const void* queries, rago_dtype query_dtype, int32_t nq, float* out_scores,
                                      void* cuda_stream) {
    Q4Rows R;
    const rago_status st = q4_check(codes, scales, scale_dtype, N, d, group, queries, query_dtype, nq, &R);
    if (st != RAGO_OK) return st;
    if (N == 0 || nq == 0) return RAGO_OK;
    if (!out_scores) return fail_q4(RAGO_EINVAL, "null pointer", 0);
    if (reinterpret_cast<uintptr_t>(out_scores) % 4) return fail_q4(RAGO_EALIGN, "out_scores are not aligned to their type", 0);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int dev = 0, sms = 0, launches = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    for (int q0 = 0; q0 < nq && e == cudaSuccess; ++launches) {
        const Q4ScoresPlan P = q4_scores_plan(R, query_dtype == RAGO_BF16, nq - q0, sms);
        const int sb = scale_dtype == RAGO_BF16;
        e = group == 32 ? q4_scores_launch<1>(P, R, sb, queries, q0, dev, sms, out_scores, s)
          : group == 64 ? q4_scores_launch<2>(P, R, sb, queries, q0, dev, sms, out_scores, s)
                        : q4_scores_launch<4>(P, R, sb, queries, q0, dev, sms, out_scores, s);
        q0 += P.nq;
    }
    return q4_done(e, launches, "4-bit scores kernel");
}

extern "C" rago_status rago_q4_rescore(const uint8_t* codes, const void* scales, rago_dtype scale_dtype, int64_t N, int32_t d,
                                       int32_t group, const void* queries, rago_dtype query_dtype, int32_t nq, const int64_t* ids,
                                       int32_t k, int32_t metric, float* out_dists, void* cuda_stream) {
    Q4Rows R;
    rago_status st = q4_check(codes, scales, scale_dtype, N, d, group, queries, query_dtype, nq, &R);
    if (st == RAGO_OK) st = q4_check_lists(nq, ids, k, metric, out_dists);
    if (st != RAGO_OK || nq == 0) return st;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int sms = 0;
    cudaError_t e = q4_sms(&sms);
    if (e != cudaSuccess) return q4_done(e, 0, "4-bit rescore kernel");
    e = q4_types(query_dtype, scale_dtype, metric, [&](auto qb, auto sb, auto l2) {
        constexpr bool Q = decltype(qb)::value, S = decltype(sb)::value, L = decltype(l2)::value;
        auto launch = [&](auto kernel, int lanes) {
            // CTAs per query: enough to fill the GPU a few times over, each warp with something to do (1024 x 100 of 768: 19.1 us, 2 CTAs an
            // SM 21.5, 32 18.6)
            const int64_t most = parts_of(parts_of(k, 64 / lanes), Q4R_WARPS);
            int64_t per = parts_of(8LL * sms, nq);
            per = per < most ? per : most;
            return launch_overlapped(kernel, dim3((unsigned)nq, (unsigned)(per < 65535 ? per : 65535)), dim3(Q4R_WARPS * 32), (size_t)d * 4, s, R, queries, ids, k, out_dists);
        };
        // rows of up to 128 numbers are four lanes' work at most: 4096 x 100 of 128 16.1 us, with 8 lanes 27.0 (few candidates go the other way, 64 x 20
        // 2.0 and 1.8; of 256 numbers 27.5 and 28.6, 64 x 20 2.9 and 1.6)
        return d <= 128 ? launch(q4_rescore_kernel<Q, S, L, 2>, 2) : launch(q4_rescore_kernel<Q, S, L, 8>, 8);
    });
    return q4_done(e, 1, "4-bit rescore kernel");
}

extern "C" rago_status rago_q4_rescore_backward(const uint8_t* codes, const void* scales, rago_dtype scale_dtype, int64_t N, int32_t d,
                                                int32_t group, const void* queries, rago_dtype query_dtype, int32_t nq,
                                                const int64_t* ids, int32_t k, int32_t metric, const float* grad_dists,
                                                void* grad_queries, void* cuda_stream) {
    Q4Rows R;
    rago_status st = q4_check(codes, scales, scale_dtype, N, d, group, queries, query_dtype, nq, &R);
    if (st == RAGO_OK) st = q4_check_lists(nq, ids, k, metric, grad_dists);
    if (st != RAGO_OK || nq == 0) return st;
    if (!grad_queries) return fail_q4(RAGO_EINVAL, "null pointer", 0);
    if (reinterpret_cast<uintptr_t>(grad_queries) % 16) return fail_q4(RAGO_EALIGN, "grad_queries need 16-byte alignment", 0);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int sms = 0;
    cudaError_t e = q4_sms(&sms);
    if (e != cudaSuccess) return q4_done(e, 0, "4-bit rescore backward kernel");
    // About 256 threads: 1024 x 100 of 768 26.5 us, with 128 37.5, with 512 31.5 (rows of 128 would rather have 128: 4096 x 100 22 instead of 33).
    // Clusters while the queries do not fill the GPU and a team has 8 candidates left: 1 x 200 of 768 4.6 us, without 12.1; 16 x 500 of 1024
    // 8.6 and 33.0.
    const int per_row = d / 16, teams = per_row >= 256 ? 1 : 256 / per_row, threads = (teams * per_row + 31) / 32 * 32;  // at most 512
    int cluster_log2 = 0;
    while ((1 << cluster_log2) < Q4B_MAX_CLUSTER && (int64_t)nq << cluster_log2 < 2 * sms && k >= (int64_t)(8 * teams) << cluster_log2) ++cluster_log2;
    const int cluster = 1 << cluster_log2;
    const size_t smem = (size_t)(teams + (metric == RAGO_L2 ? 1 : 0)) * d * 4;  // the teams' sums, the query: at most 64 KB
    e = q4_types(query_dtype, scale_dtype, metric, [&](auto qb, auto sb, auto l2) {
        auto kernel = q4_rescore_backward_kernel<decltype(qb)::value, decltype(sb)::value, decltype(l2)::value>;
        if (smem > 40 * 1024) {  // long rows; 48 KB go without asking, some of them to the kernel's own arrays
            const cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (r != cudaSuccess) return r;
        }
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((int64_t)nq * cluster)); cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
        cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
        return cudaLaunchKernelEx(&cfg, kernel, R, queries, ids, (int)k, grad_dists, teams, cluster_log2, grad_queries);
    });
    return q4_done(e, 1, "4-bit rescore backward kernel");
}
