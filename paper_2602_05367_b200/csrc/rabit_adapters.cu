// Low-rank adapters of many requests beside a layer, and the gradients of their factors.
//
//   u[t] = A[id_t] x[t],   y[t] = layer(x[t]) + scale[id_t] * B[id_t]^T u[t]
//   da[i] = scale[i] * sum_{t: id_t = i} p[t] x[t]^T,   db[i] = scale[i] * sum_{t: id_t = i} u[t] dy[t]^T
//
// Every factor is `rank` rows along a side of the layer, so both products of the forward pass and of the input gradient are the same kernels: narrow_kernel (a
// side to the rank) beside the layer and widen_kernel (the rank to a side) behind it, or decode_kernel, both in one, for few rows; the gradients are
// factor_kernel.  All are MMAs of mma.sync: their products are a few per cent of the layer's, their inner or outer size is the rank (1 to 128),
// and what bounds them is memory, latency or the instructions around the MMAs, not the tensor pipe (mma.sync reaches 537 TFLOP/s here).
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstring>

#include "rabit_internal.h"

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxGroup = 8;                           // layers in one launch
// Checked build (-DRABIT_CHECKED, python paper_2602_05367_b200/build.py --checked): every address that is made from ids, lists of rows or sizes is compared with
// its buffer first; a violation sets the word that rabit_selftest_index_faults reads, and the access is skipped.  In the ordinary build the checks compile to nothing.
#ifdef RABIT_CHECKED
__device__ unsigned int g_index_fault;
#define RABIT_IN_RANGE(cond) ((cond) ? true : (atomicExch(&g_index_fault, 1u), false))
// whether `bytes` bytes at p lie in the `size` bytes at base
__device__ __forceinline__ bool inside(const void* p, size_t bytes, const void* base, size_t size) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), from = reinterpret_cast<uintptr_t>(base);
    return at >= from && at + bytes <= from + size;
}
#else
#define RABIT_IN_RANGE(cond) true
#endif

constexpr int kMostRows = 0x7FFFFF00;                  // rows of a call: a tile's places behind the last one are 32-bit numbers too

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same on top of zero
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// fp32 operands of MMAs with fp16 ones.  Values that share a power of two are scaled so that the largest lies in [2^14, 2^15), then each is the sum of two fp16
// values: 22 bits of it, or all bits down to 2^-39 of the largest where that is less.  (tf32 MMAs, two per operand part, have twice the number for the
// same products, and their fp16 operand has to be converted: 4096 x 11008, rank 64, 4096 tokens took 150 us for the gradients and 118 for widen_kernel.)
__device__ __forceinline__ void range_of(float largest, float& to, float& back) {   // to * largest in [2^14, 2^15); back = 1 / to
    const uint32_t e = max(__float_as_uint(largest) >> 23, 15u);
    to = __uint_as_float((268u - e) << 23);
    back = __uint_as_float((e - 14u) << 23);
}
__device__ __forceinline__ float finite_size(float v) {                         // |v|; 0 for what has no size
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? __uint_as_float(b) : 0.f;
}
__device__ __forceinline__ void split_f16(float v, float to, __half& hi, __half& lo) {
    v *= to;
    hi = __float2half_rn(v);
    const float rest = v - __half2float(hi);
    lo = __float2half_rn(finite_size(v) == fabsf(v) ? rest : 0.f);              // (an infinity has no rest, a NaN is one in hi)
}
__device__ __forceinline__ float2 floats_of(uint32_t pair) { return __half22float2(*reinterpret_cast<const __half2*>(&pair)); }

constexpr int kMaxCluster = 8;
// Elements 4 e .. 4 e + 3 of `values` (the same place in every CTA of the cluster), added up in the order of the CTAs.  The loads go out together: one after
// the other they were most of the time of the kernels below.
__device__ __forceinline__ float4 cluster_sum(const cg::cluster_group& cluster, float* values, int parts, int e) {
    float4 v[kMaxCluster];
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q) v[q] = q < parts ? reinterpret_cast<const float4*>(cluster.map_shared_rank(values, q))[e] : make_float4(0.f, 0.f, 0.f, 0.f);
    float4 s = v[0];
#pragma unroll
    for (int q = 1; q < kMaxCluster; ++q) {
        s.x += v[q].x; s.y += v[q].y; s.z += v[q].z; s.w += v[q].w;
    }
    return s;
}
// Four neighbours of a row of u (or of a gradient) to memory, of which those before `n` exist
__device__ __forceinline__ void store_4(float* at, const float4& v, int n, bool fours) {
    if (fours) {
        *reinterpret_cast<float4*>(at) = v;
    } else {
        if (n > 0) at[0] = v.x;
        if (n > 1) at[1] = v.y;
        if (n > 2) at[2] = v.z;
        if (n > 3) at[3] = v.w;
    }
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// ---- u[t] = A[id_t] x[t] -----------------------------------------------------------------------------------

struct NarrowLayer {
    const __half *x, *a;
    float* u;
    int n, rank, count;
};
struct NarrowParams {
    NarrowLayer layer[kMaxGroup];
    const int* ids;
    int batch, beside;                                                          // beside: the kernel before this one is the layer's, still running
    int shares;                                                                 // clusters that share the adapters of a tile of rows; the later ones are mostly idle, so they come last
};

// ---- asynchronous copies to shared memory --------------------------------------------------------------------

__device__ __forceinline__ void copy_async_16(void* dst, const void* src, bool valid) {   // (not valid: zeros)
    const uint32_t size = valid ? 16u : 0u;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(size) : "memory");
}
__device__ __forceinline__ void copy_async_4(void* dst, const void* src, bool valid) {
    const uint32_t size = valid ? 4u : 0u;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(size) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// 8 halves at any place, of which those before `n` are inside their row, from the one or two aligned 16-byte pieces that hold them
__device__ __forceinline__ uint4 extract_8(const uint4& lo, const uint4& hi, const __half* src, int n) {
    const uint32_t skip = (uint32_t)(reinterpret_cast<uintptr_t>(src) >> 1) & 7u;   // halves of the first piece before src
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = skip & 4u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = skip & 2u ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = skip & 1u ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
        if (n < 8) w[i] = 2 * i + 1 < n ? w[i] : 2 * i < n ? w[i] & 0xFFFFu : 0u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Both pieces to shared memory (`second` 16-byte units apart), asynchronously: what lies beyond `end`, the end of the buffer, or is not needed arrives as zeros and is
// not read.
__device__ __forceinline__ void copy_async_pieces(uint4* dst, int second, const __half* src, int n, const __half* begin, const __half* end) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(src), piece = at & ~(uintptr_t)15, last = reinterpret_cast<uintptr_t>(end);
    const bool two = n > 0 && (int)((at >> 1) & 7u) + min(n, 8) > 8;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uintptr_t from = piece + 16 * h;
        uint32_t size = (h == 0 ? n > 0 : two) ? (uint32_t)min((long long)16, (long long)(last - from)) : 0u;
        if (size != 0u && !RABIT_IN_RANGE(size <= 16u && inside(reinterpret_cast<const void*>(from), size, begin, last - reinterpret_cast<uintptr_t>(begin)))) size = 0u;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + h * second)), "l"(size ? from : piece), "r"(size) : "memory");
    }
}
// The same straight from memory, for rows of any length; `end` is the end of the buffer, which starts on 16 bytes: halves one by one where a piece would reach beyond it.
__device__ __forceinline__ uint4 load_8(const __half* src, int n, const __half* begin, const __half* end) {
    if (n <= 0) return make_uint4(0u, 0u, 0u, 0u);
    if (!RABIT_IN_RANGE(inside(src, 2 * min(n, 8), begin, reinterpret_cast<const char*>(end) - reinterpret_cast<const char*>(begin)) && (reinterpret_cast<uintptr_t>(begin) & 15u) == 0u)) return make_uint4(0u, 0u, 0u, 0u);
    const uintptr_t at = reinterpret_cast<uintptr_t>(src);
    const uint4* piece = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
    const bool two = (int)((at >> 1) & 7u) + min(n, 8) > 8;
    if (reinterpret_cast<const __half*>(piece + (two ? 2 : 1)) > end) {
        uint32_t v[4] = {};
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < n) v[q >> 1] |= (uint32_t)__half_as_ushort(src[q]) << (16 * (q & 1));
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    return extract_8(piece[0], two ? piece[1] : make_uint4(0u, 0u, 0u, 0u), src, n);
}
// 8 halves to dst, those before `n`.  VEC: dst lies on 16 bytes and all are inside.  Otherwise in words of the 4-byte grid, with a half before and behind them where dst is odd.
template <bool VEC>
__device__ __forceinline__ void store_8(__half* dst, int n, const uint32_t (&v)[4]) {
    if constexpr (VEC) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
        const bool odd = (reinterpret_cast<uintptr_t>(dst) & 2u) != 0u;
        if (n < 8) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < n) dst[q] = __ushort_as_half((unsigned short)(v[q >> 1] >> (16 * (q & 1))));
        } else if (odd) {
            dst[0] = __ushort_as_half((unsigned short)v[0]);
#pragma unroll
            for (int i = 0; i < 3; ++i) *reinterpret_cast<uint32_t*>(dst + 1 + 2 * i) = __funnelshift_r(v[i], v[i + 1], 16);
            dst[7] = __ushort_as_half((unsigned short)(v[3] >> 16));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(dst + 2 * i) = v[i];
        }
    }
}

// A cluster takes a tile of 16 * WM rows; 8 / WM groups of WM warps side by side and the CTAs of the cluster cut the contraction into parts, which meet in shared
// memory, then over the cluster, in a fixed order.  Products are m16n8k16 MMAs of fp16 operands, rows by ranks.  x and the factor come through a ring of
// asynchronous copies, 64 columns (a line of memory) per group of warps and stage.  The order of a contraction is free, so a lane takes 8 consecutive columns
// of each of its rows (one 16-byte read) as the four operand words of two MMAs.
// Rows of different adapters in one tile: the tile is multiplied with each adapter that occurs, and a row keeps the products of its own; warps without rows of an
// adapter sit it out.  Several clusters share the adapters of a tile.
// The tensor core truncates when it accumulates: after 16 MMAs the sums go to other registers.
// Bound: x from memory; from rank 64 on shared memory, which every warp reads the whole factor from for its 16 rows.  4096 rows of 4096 columns, rank 16: 14 us (33.5 MB
// of x: 5.1 at the copy rate, then the start and the sum over the cluster, 2 us each); rank 64: 31 us, 1037 rows of 14336 columns: 31.
template <int NR, int WM>
struct Narrow {
    static constexpr int kRows = 16 * WM, kRanks = 8 * NR, WK = kWarps / WM;
    static constexpr int kABytes = WK * kRanks * 128, kStageBytes = kABytes + kWarps * 4 * 32 * 16;
    static constexpr int kPerSm = NR <= 8 ? 2 : 1, kFit = 226 * 1024 / kPerSm / kStageBytes, kStages = kFit < 4 ? kFit : 4;
    static constexpr int kBytes = kStages * kStageBytes;
    static_assert(WK * kRows * kRanks * 4 <= kBytes && kPerSm * (kBytes + 1024) <= 228 * 1024 && kBytes <= 227 * 1024, "the sums fit, and so many CTAs per SM");
};
template <int NR, int WM>
__global__ void __launch_bounds__(kThreads, (Narrow<NR, WM>::kPerSm)) narrow_kernel(const __grid_constant__ NarrowParams P) {
    using T = Narrow<NR, WM>;
    extern __shared__ __align__(16) unsigned char smem[];
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, tq = lane & 3, wm = warp % WM, wk = warp / WM;
    const NarrowLayer& L = P.layer[blockIdx.z];
    const int share = blockIdx.y, tile0 = (int)(blockIdx.x / parts) * T::kRows, n = L.n, rank = L.rank, row0 = tile0 + 16 * wm;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!P.beside) asm volatile("griddepcontrol.wait;" ::: "memory");

    // rows of the tile lane by lane, 32 to a word
    constexpr int kWords = (T::kRows + 31) / 32;
    int id[kWords];
    uint32_t left[kWords], mine[kWords], named[kWords];
    bool any = false;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const int r = 32 * w + lane;
        id[w] = r < T::kRows && tile0 + r < P.batch ? __ldcg(P.ids + tile0 + r) : -1;   // (from L2: beside the layer nothing has made L1 forget an earlier call's)
        if (id[w] >= L.count) id[w] = -1;
        named[w] = left[w] = __ballot_sync(0xFFFFFFFFu, id[w] >= 0);
        mine[w] = 0u;
        any = any || left[w] != 0u;
    }
    const int chunks = (n + 63) / 64;
    const int c0 = (int)((long long)chunks * part / parts), c1 = (int)((long long)chunks * (part + 1) / parts), iters = (c1 - c0 + T::WK - 1) / T::WK;
    float sum[NR][4] = {};
    int turn = 0;
    for (; any; ++turn) {
        int cur = -1;
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            const int v = __shfl_sync(0xFFFFFFFFu, id[w], left[w] ? __ffs(left[w]) - 1 : 0);
            if (cur < 0 && left[w]) cur = v;
        }
        uint32_t own = 0u;                                                      // of this warp's 16 rows
        any = false;
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            const uint32_t match = __ballot_sync(0xFFFFFFFFu, id[w] == cur);
            left[w] &= ~match;
            any = any || left[w] != 0u;
            if (turn % P.shares == share) {
                mine[w] |= match;
                if (w == wm / 2) own = (match >> (16 * (wm & 1))) & 0xFFFFu;
            }
        }
        if (turn % P.shares != share) continue;
        const bool has[2] = {(own >> gq & 1u) != 0u, (own >> (8 + gq) & 1u) != 0u};
        const __half* a = L.a + (size_t)cur * rank * n;
        // What a thread copies lies at fixed places of a stage: 16-byte pieces of the factor's rows, 8 to a row and group of warps (odd rows have their two halves
        // exchanged, for the banks), and pieces of its warp's rows of x.
        constexpr int kCopies = (T::WK * T::kRanks * 8 + kThreads - 1) / kThreads;
        const int piece = threadIdx.x & 7, j0 = threadIdx.x >> 3;
        const bool all_copy = T::WK * T::kRanks * 8 >= kThreads || (int)threadIdx.x < T::WK * T::kRanks * 8;
        const __half* a0 = a + (size_t)(j0 % T::kRanks) * n + (c0 + j0 / T::kRanks) * 64 + piece * 8;
        const int x_row = lane >> 3;                                            // of four rows to a copy of the warp: 128 bytes of each, whole lines
        const __half* x0 = L.x + (size_t)(row0 + x_row) * n + (size_t)(c0 + wk) * 64 + (lane & 7) * 8;
        const size_t rows32 = (size_t)32 * n, rows4 = (size_t)4 * n;
        auto fetch = [&](int it) {
            unsigned char* stage = smem + it % T::kStages * T::kStageBytes;
            if (it < iters) {
                const int chunk0 = c0 + it * T::WK;
                const bool whole = chunk0 + T::WK <= c1 && (chunk0 + T::WK) * 64 <= n;   // (all but the last)
                if (all_copy) {
#pragma unroll
                    for (int i = 0; i < kCopies; ++i) {
                        constexpr int kPer = T::kRanks >= 32 ? T::kRanks / 32 : 1;      // copies of 32 rows to a group of warps
                        const int k = T::kRanks >= 32 ? i / kPer : i * (32 / T::kRanks) + j0 / T::kRanks, j = (T::kRanks >= 32 ? i % kPer * 32 : 0) + j0 % T::kRanks;
                        const bool in = j < rank && (whole || (chunk0 + k < c1 && (chunk0 + k) * 64 + piece * 8 < n));
                        const __half* src = a0 + (size_t)it * (T::WK * 64) + (T::kRanks >= 32 ? (size_t)(i % kPer) * rows32 + i / kPer * 64 : (size_t)(i * (32 / T::kRanks) * 64));
                        unsigned char* dst = stage + (k * T::kRanks + j) * 128 + ((piece ^ ((j & 1) << 2)) << 4);
                        if (RABIT_IN_RANGE(inside(dst, 16, stage, T::kABytes) && (!in || inside(src, 16, L.a, (size_t)L.count * rank * n * 2)))) copy_async_16(dst, in ? src : L.a, in);
                    }
                }
                if (own != 0u) {
                    const __half* src = x0 + (size_t)it * (T::WK * 64);
                    const bool col_in = whole || (chunk0 + wk < c1 && (chunk0 + wk) * 64 + (lane & 7) * 8 < n);
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const int r = 4 * m + x_row;
                        const bool in = col_in && (own >> r & 1u);
                        unsigned char* dst = stage + T::kABytes + (warp * 16 + r) * 128 + (((lane & 7) ^ ((r & 1) << 2)) << 4);
                        if (RABIT_IN_RANGE(inside(dst, 16, stage, T::kStageBytes) && (!in || inside(src + m * rows4, 16, L.x, (size_t)P.batch * n * 2)))) copy_async_16(dst, in ? src + m * rows4 : L.x, in);
                    }
                }
            }
            copy_async_commit();
        };
#pragma unroll
        for (int it = 0; it < T::kStages - 1; ++it) fetch(it);
        float acc[NR][4] = {};
        auto flush = [&]() {
#pragma unroll
            for (int j = 0; j < NR; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (has[e >> 1]) sum[j][e] += acc[j][e];
                    acc[j][e] = 0.f;
                }
        };
        for (int it = 0; it < iters; ++it) {
            copy_async_wait<T::kStages - 2>();
            __syncthreads();                                                    // everybody's copies of this stage are there, and the slot of the one before is free
            fetch(it + T::kStages - 1);
            if (own == 0u) continue;
            const unsigned char* stage = smem + it % T::kStages * T::kStageBytes;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int swizzled = ((s ^ (gq & 1)) << 6) + tq * 16;
                const unsigned char *x_at = stage + T::kABytes + (warp * 16 + gq) * 128 + swizzled, *at = stage + (wk * T::kRanks + gq) * 128 + swizzled;
                const uint4 x0 = *reinterpret_cast<const uint4*>(x_at), x1 = *reinterpret_cast<const uint4*>(x_at + 8 * 128);
#pragma unroll
                for (int j0 = 0; j0 < NR; j0 += 8) {                            // (products on top of one another far apart: an MMA takes about four others' time to finish)
                    constexpr int kJ = NR < 8 ? NR : 8;
                    uint4 w[kJ];
#pragma unroll
                    for (int j = 0; j < kJ; ++j) w[j] = *reinterpret_cast<const uint4*>(at + (j0 + j) * 8 * 128);
#pragma unroll
                    for (int j = 0; j < kJ; ++j) mma_f16(acc[j0 + j], x0.x, x1.x, x0.y, x1.y, w[j].x, w[j].y);
#pragma unroll
                    for (int j = 0; j < kJ; ++j) mma_f16(acc[j0 + j], x0.z, x1.z, x0.w, x1.w, w[j].z, w[j].w);
                }
            }
            if (it % 4 == 3) flush();
        }
        flush();
        copy_async_wait<0>();
        __syncthreads();                                                        // (the next adapter fills the same stages)
    }
    bool taken = share == 0;                                               // rows without adapter: u is zero, the first cluster's
#pragma unroll
    for (int w = 0; w < kWords; ++w) taken = taken || mine[w] != 0u;
    if (!taken) return;                                                         // (the whole cluster agrees)
    float* red = reinterpret_cast<float*>(smem);                                // [WK][kRows][kRanks]
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        float* at = red + ((size_t)wk * T::kRows + 16 * wm + gq) * T::kRanks + 8 * j + 2 * tq;
        *reinterpret_cast<float2*>(at) = make_float2(sum[j][0], sum[j][1]);
        *reinterpret_cast<float2*>(at + 8 * T::kRanks) = make_float2(sum[j][2], sum[j][3]);
    }
    if (T::WK > 1) {
        __syncthreads();
        for (int e = threadIdx.x; e < T::kRows * T::kRanks; e += kThreads) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < T::WK; ++w) s += red[w * T::kRows * T::kRanks + e];
            red[e] = s;
        }
    }
    cluster.sync();
    for (int e = part * kThreads + threadIdx.x; e < T::kRows * T::kRanks / 4; e += parts * kThreads) {
        const int row = e / (T::kRanks / 4), j = e % (T::kRanks / 4) * 4;
        uint32_t word = 0u;
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            if (row / 32 == w) word = mine[w] | (share == 0 ? ~named[w] : 0u);
        if (j >= rank || tile0 + row >= P.batch || !((word >> (row & 31)) & 1u)) continue;
        float* to = L.u + (size_t)(tile0 + row) * rank + j;
        if (RABIT_IN_RANGE(inside(to, 4 * min(rank - j, 4), L.u, (size_t)P.batch * rank * 4))) store_4(to, cluster_sum(cluster, red, parts, e), rank - j, rank % 4 == 0);
    }
    cluster.sync();
    // One CTA, whose share is always taken, waits for the layer: the grid ends behind the layer's, so what waits for this one has y.  The others make room.
    if (P.beside && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---- y[t] += scale[id_t] * B[id_t]^T u[t] --------------------------------------------------------------------

struct WidenLayer {
    const __half* b;
    const float *u, *scale;
    __half* y;
    int m, rank, count;
};
struct WidenParams {
    WidenLayer layer[kMaxGroup];
    const int* ids;
    int batch, beside;                                                          // as in NarrowParams
    int blocks;                                                                 // row blocks of a CTA, one after the other
};
// 16-byte pieces of a row (pair) of u as operand: half as many again are 4 more than a multiple of 8 from pair to pair, so that two pairs that a load touches, 64
// bytes each, meet in no bank
__host__ __device__ constexpr int operand_stride(int fours) { return fours + 2; }
constexpr int kWidenRows = 32;
// u as operand of an MMA of 16 rows and 16 ranks: four registers that lie behind one another, ranks 4 tq, 4 tq + 1 of row gq and of row gq + 8, then the two ranks
// behind those; one 16-byte piece in shared memory for the first parts, `kPair` pieces further one for the second (put together in registers, every
// operand would cost four moves).  [pair of rows][first, second][ranks / 4], the pairs of a 16-row tile 8 to a block.
template <int R16>
struct Operand {
    static constexpr int kFours = 4 * R16, kSecond = operand_stride(kFours), kPair = 2 * kSecond;
    static __host__ __device__ constexpr int pieces(int rows) { return rows / 2 * kPair; }
    // where rows `row` and row ^ 8 lie
    static __device__ __forceinline__ int at(int row) { return ((row >> 4) * 8 + (row & 7)) * kPair; }
};
// Four neighbours of row `row` of u, whose other parts the next kFours - 1 lanes hold, into the operand.  Returns the factor that takes products back.
template <int R16>
__device__ __forceinline__ float split_row(uint4* operand, int row, int four, const float4& v) {
    using O = Operand<R16>;
    float largest = fmaxf(fmaxf(finite_size(v.x), finite_size(v.y)), fmaxf(finite_size(v.z), finite_size(v.w)));
#pragma unroll
    for (int d = 1; d < O::kFours; d <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, d));
    float to, back;
    range_of(largest, to, back);
    __half h[4], l[4];
    split_f16(v.x, to, h[0], l[0]);
    split_f16(v.y, to, h[1], l[1]);
    split_f16(v.z, to, h[2], l[2]);
    split_f16(v.w, to, h[3], l[3]);
    __half2* hi = reinterpret_cast<__half2*>(operand + O::at(row) + four) + ((row >> 3) & 1);
    __half2* lo = hi + 4 * O::kSecond;
    hi[0] = __halves2half2(h[0], h[1]);
    hi[2] = __halves2half2(h[2], h[3]);
    lo[0] = __halves2half2(l[0], l[1]);
    lo[2] = __halves2half2(l[2], l[3]);
    return back;
}
// 16 rows by GROUPS * 32 columns by 16 ranks: `u` the lane's piece of the operand, `second` pieces further its second part; f the factor's fragments of the groups' four
// column tiles: ranks 4 tq and 4 tq + 1, the two behind them.
template <int GROUPS>
__device__ __forceinline__ void widen_step(float (&acc)[GROUPS][4][4], bool first, const uint4* u, int second, const uint32_t (&f)[GROUPS][4][2]) {
    const uint4 a = u[0], b = u[second];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (first) mma_f16_first(acc[g][q], a.x, a.y, a.z, a.w, f[g][q][0], f[g][q][1]);
            else mma_f16(acc[g][q], a.x, a.y, a.z, a.w, f[g][q][0], f[g][q][1]);
        }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int q = 0; q < 4; ++q) mma_f16(acc[g][q], b.x, b.y, b.z, b.w, f[g][q][0], f[g][q][1]);
}
template <int R16, bool VEC>
struct Widen {
    static constexpr int kRanks = 16 * R16, kTiles = kWidenRows / 16, kFours = kRanks / 4;
    static constexpr int kGroups = R16 <= 2 && VEC ? 2 : 1, kCols = 32 * kGroups * kWarps;      // of 32 columns to a warp
    static constexpr int kLanes = 4 * kGroups, kBlockPieces = kWidenRows * kLanes;   // 16-byte pieces of a warp's row of y, of its block
    // place of piece p of row r: two rows that a load touches, 64 bytes each, meet in no bank
    static __device__ __forceinline__ int piece(int r, int p) { return r * kLanes + (kLanes == 8 ? p ^ ((r & 1) << 2) : p); }
    static constexpr int kPlanes = VEC ? 1 : 2, kRingBytes = 2 * kPlanes * kWarps * kBlockPieces * 16, kUBytes = kWidenRows * kRanks * 4;
    static constexpr int kBytes = kRingBytes + kUBytes + Operand<R16>::pieces(kWidenRows) * 16 + kWidenRows * 4;
    static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two CTAs per SM");
};
// Row gq (h = 0) or gq + 8 (h = 1) of those products on top of the 8 columns of y that were read as `old`.  The layer's sum is there in fp16, rounded by the layer's own kernel:
// every GEMV and GEMM writes its y so, and the call has no other memory for it (fp32 would be twice the bytes of y, out and in again).  Against one rounding of the whole that costs 0.00029 of the
// largest output for 0.00021, and what is infinite there stays so.
template <bool VEC>
__device__ __forceinline__ void widen_store(__half* y, int n, const uint4& old, const float (&acc)[4][4], int h, float scale) {
    uint32_t v[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 was = floats_of(v[q]);
        const __half2 r = __floats2half2_rn(fmaf(scale, acc[q][2 * h], was.x), fmaf(scale, acc[q][2 * h + 1], was.y));
        v[q] = *reinterpret_cast<const uint32_t*>(&r);
    }
    store_8<VEC>(y, n, v);
}

struct DecodeLayer {
    const __half *x, *a, *b;
    const float* scale;
    float* u;
    __half* y;
    int n, m, rank, count;
};
struct DecodeParams {
    DecodeLayer layer[kMaxGroup];
    const int* ids;
    int batch, beside;                                                          // as in NarrowParams
};
constexpr int kDecodeRows = 1024, kWindow = 64;                                 // most rows of a batch; of those whose rows of an adapter are put together

// A CTA takes 512 columns (256 beyond rank 32), a warp 64 (32) of them, and blocks of 32 rows one after the other: rows by columns as m16n8k16 MMAs over the rank, the
// factor's fragments in registers for all rows, a row of u as two fp16 parts of a common power of two.  The order of columns in MMA tiles and of ranks is
// free: a lane's results are 8 consecutive columns of a row (one 16-byte access to y), its factor entries come from 16-byte loads, its u entries
// are four consecutive ones.  A row belongs to one adapter, so y is read and written once; y, u and ids of the next block are on their way while this
// one is multiplied (copies to shared memory: registers do not hold enough of y for the latency).
// Bound: y, in and out; the instructions around the MMAs are as many as that leaves room for, which is why a warp takes 64 columns.  4096 rows of 11008 columns,
// rank 16: 32 us (180 MB, 5.6 TB/s; with 32 columns to a warp 43, with y in registers only 51); rank 64 (32 columns to a warp, 64 spill): 74, of which 22 are MMAs.
template <int R16, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) widen_kernel(const __grid_constant__ WidenParams P) {
    using W = Widen<R16, VEC>;
    using O = Operand<R16>;
    constexpr int kTiles = W::kTiles, G = W::kGroups;
    extern __shared__ __align__(16) unsigned char widen_smem[];                 // rings of y | a block of u | the same as operand | its rows' factors
    uint4* ring = reinterpret_cast<uint4*>(widen_smem);
    float* u_block = reinterpret_cast<float*>(widen_smem + W::kRingBytes);
    uint4* us = reinterpret_cast<uint4*>(widen_smem + W::kRingBytes + W::kUBytes);
    float* backs = reinterpret_cast<float*>(us + O::pieces(kWidenRows));
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, tq = lane & 3;
    const WidenLayer& L = P.layer[blockIdx.z];
    const int col0 = blockIdx.x * W::kCols + warp * (32 * G), m_all = L.m, rank = L.rank, batch = P.batch;
    const int first_row = (int)blockIdx.y * P.blocks * kWidenRows;
    const int blocks = min(P.blocks, (batch - first_row + kWidenRows - 1) / kWidenRows);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if ((int)blockIdx.x * W::kCols >= m_all) return;
    // beside: ids and the first factor before the wait (from L2, as in narrow_kernel; without 16-byte pieces the factor comes through L1, so behind it)
    const bool early = VEC && P.beside;
    if (!early) asm volatile("griddepcontrol.wait;" ::: "memory");

    const __half* y_end = L.y + (size_t)batch * m_all;
    const bool fours = rank % 4 == 0;
    const int c = col0 + 8 * tq;                                                // the lane's columns in y: 8 here and 8 in each further group
    ring += warp * W::kBlockPieces;
    __half* y = L.y + (size_t)(first_row + gq) * m_all + c;                     // the lane's part of row gq of the block at hand
    const __half* y_from = L.y + (size_t)(first_row + lane / W::kLanes) * m_all + col0 + lane % W::kLanes * 8;   // what it copies first
    const size_t eight = (size_t)8 * m_all;
    // u of a block and the lane's part of y of the same rows: one group of copies
    auto fetch = [&](int blk, const __half* from) {
        const int row0 = first_row + blk * kWidenRows;
        if (blk < blocks) {
            // rows of 8 * kLanes columns, kLanes lanes side by side: whole lines of memory where a warp has 64 columns
            uint4* dst = ring + (blk & 1) * (W::kPlanes * kWarps * W::kBlockPieces);
#pragma unroll
            for (int t = 0; t < kWidenRows; t += 32 / W::kLanes) {
                const int r = t + lane / W::kLanes, p = lane % W::kLanes, cols = m_all - col0 - 8 * p;
                const bool in = row0 + r < batch && cols > 0;
                const __half* src = in ? from + (size_t)t * m_all : L.y;
                if (!RABIT_IN_RANGE(inside(dst + W::piece(r, p), 16, ring, W::kRingBytes - warp * W::kBlockPieces * 16) && (!in || inside(src, 2 * min(cols, 8), L.y, (size_t)batch * m_all * 2)))) continue;
                if (VEC) copy_async_16(dst + W::piece(r, p), src, in);
                else copy_async_pieces(dst + W::piece(r, p), kWarps * W::kBlockPieces, src, in ? cols : 0, L.y, y_end);
            }
            for (int i = threadIdx.x; i < kWidenRows * W::kFours; i += kThreads) {
                const int r = i / W::kFours, j = i % W::kFours * 4;
                const float* src = L.u + (size_t)(row0 + r) * rank + j;
                const bool in = row0 + r < batch;
                float* to = u_block + 4 * i;
                if (in && j < rank && !RABIT_IN_RANGE(inside(src, 4 * min(rank - j, 4), L.u, (size_t)batch * rank * 4))) continue;
                if (fours) {
                    copy_async_16(to, in && j < rank ? src : L.u, in && j < rank);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) copy_async_4(to + q, in && j + q < rank ? src + q : L.u, in && j + q < rank);
                }
            }
        }
        copy_async_commit();
    };
    auto load_id = [&](int blk) {
        const int r = first_row + blk * kWidenRows + lane, v = blk < blocks && r < batch ? __ldcg(P.ids + r) : -1;
        return v < L.count ? v : -1;
    };
    uint32_t f[R16][G][4][2];                                                   // [16 ranks][32 columns][column tile]: ranks 4 tq and 4 tq + 1, the two behind them
    auto load_factor = [&](int cur) {
        const uint32_t pick = gq & 1 ? 0x7632u : 0x5410u;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int cf = col0 + 32 * g + 8 * (gq >> 1);
            const __half* b = L.b + ((size_t)cur * rank + 4 * tq) * m_all + cf;
#pragma unroll
            for (int k = 0; k < R16; ++k) {
                if constexpr (VEC) {
                    uint4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = 16 * k + 4 * tq + i < rank && cf < m_all && RABIT_IN_RANGE(inside(b + (size_t)(16 * k + i) * m_all, 16, L.b, (size_t)L.count * rank * m_all * 2)) ? __ldcg(reinterpret_cast<const uint4*>(b + (size_t)(16 * k + i) * m_all)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        f[k][g][0][p] = __byte_perm(v[2 * p].x, v[2 * p + 1].x, pick);
                        f[k][g][1][p] = __byte_perm(v[2 * p].y, v[2 * p + 1].y, pick);
                        f[k][g][2][p] = __byte_perm(v[2 * p].z, v[2 * p + 1].z, pick);
                        f[k][g][3][p] = __byte_perm(v[2 * p].w, v[2 * p + 1].w, pick);
                    }
                } else {                                                        // the halves that the fragments hold
                    uint32_t v[4][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned short* row = reinterpret_cast<const unsigned short*>(b + (size_t)(16 * k + i) * m_all) + (gq & 1);
#pragma unroll
                        for (int q = 0; q < 4; ++q) v[i][q] = 16 * k + 4 * tq + i < rank && cf + 2 * q + (gq & 1) < m_all && RABIT_IN_RANGE(inside(row + 2 * q, 2, L.b, (size_t)L.count * rank * m_all * 2)) ? row[2 * q] : 0u;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int p = 0; p < 2; ++p) f[k][g][q][p] = v[2 * p][q] | v[2 * p + 1][q] << 16;
                }
            }
        }
    };

    if (!early) fetch(0, y_from);
    int next_id = load_id(0), held = -1;                                        // held: the adapter whose factor the registers hold
    if (early) {
        const uint32_t named = __ballot_sync(0xFFFFFFFFu, next_id >= 0);
        if (named) load_factor(held = __shfl_sync(0xFFFFFFFFu, next_id, __ffs(named) - 1));
        asm volatile("griddepcontrol.wait;" ::: "memory");
        fetch(0, y_from);
    }
    for (int blk = 0; blk < blocks; ++blk) {
        const int id = next_id;
        uint32_t left = __ballot_sync(0xFFFFFFFFu, id >= 0);
        int cur = left ? __shfl_sync(0xFFFFFFFFu, id, __ffs(left) - 1) : held;
        if (cur != held) load_factor(held = cur);
        next_id = load_id(blk + 1);
        copy_async_wait<0>();
        __syncthreads();                                                        // this block is there, and nobody reads the one before any more
        for (int i = threadIdx.x; i < kWidenRows * W::kFours; i += kThreads) {
            const float back = split_row<R16>(us, i / W::kFours, i % W::kFours, reinterpret_cast<const float4*>(u_block)[i]);
            if (i % W::kFours == 0) backs[i / W::kFours] = back;
        }
        __syncthreads();
        y_from += 4 * eight;
        fetch(blk + 1, y_from);
        const uint4* old = ring + (blk & 1) * (W::kPlanes * kWarps * W::kBlockPieces);
        while (left != 0u) {
            if (cur != held) load_factor(held = cur);
            const uint32_t match = __ballot_sync(0xFFFFFFFFu, id == cur);
            left &= ~match;
            const float scale = RABIT_IN_RANGE(cur >= 0 && cur < L.count) ? __ldcg(L.scale + cur) : 0.f;
#pragma unroll
            for (int mt = 0; mt < kTiles; ++mt) {
                const uint32_t hits = (match >> (16 * mt)) & 0xFFFFu;
                if (hits == 0u) continue;
                float acc[G][4][4];
#pragma unroll
                for (int k = 0; k < R16; ++k) widen_step<G>(acc, k == 0, us + O::at(16 * mt + gq) + 4 * k + tq, O::kSecond, f[k]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!((hits >> (8 * h + gq)) & 1u)) continue;
                    const float factor = scale * backs[16 * mt + 8 * h + gq];
#pragma unroll
                    for (int g = 0; g < G; ++g)
                        if (c + 32 * g < m_all) {
                            __half* to = y + (2 * mt + h) * eight + 32 * g;
                            const uint4* was = old + W::piece(16 * mt + 8 * h + gq, 4 * g + tq);
                            if (!RABIT_IN_RANGE(inside(to, 2 * min(m_all - c - 32 * g, 8), L.y, (size_t)batch * m_all * 2))) continue;
                            widen_store<VEC>(to, m_all - c - 32 * g, VEC ? *was : extract_8(was[0], was[(W::kPlanes - 1) * kWarps * W::kBlockPieces], to, m_all - c - 32 * g), acc[g], h, factor);
                        }
                }
            }
            if (left != 0u) cur = __shfl_sync(0xFFFFFFFFu, id, __ffs(left) - 1);
        }
        y += 4 * eight;
    }
    copy_async_wait<0>();
}

// ---- both steps in one launch, for few rows --------------------------------------------------------------------

// Up to 1024 rows.  Behind the layer, clusters of CTAs take one adapter and up to 16 of its rows at a time: in windows of 64 rows the rows of an adapter are
// put together wherever they stand, the items being found by one match over the window.  A cluster makes u of the rows as narrow_kernel does and adds their part to y
// as widen_kernel does, the CTAs taking columns in turn.  The CTAs send their sums of u to one another, so one cluster barrier lies between the two steps; the factor's first entries
// and y of the second are fetched before it.  One launch instead of two saves a launch's latency and the way of u through memory.
// Bound: latencies (dependency wait, ids, x and factor, cluster barrier, y): few instructions on the way count, not bytes.  One token of 1024 x 4096, rank 16: 5900
// clocks, of which ids and items 810, the rank's sums 1500, their way through the cluster 1500, y 510; 3.8 us behind the layer's 2.7.  48 rows of ten
// adapters, 14336 x 4096, rank 32: 10.4 us behind 15.9 (two sets of columns on their way; with one 14).  Behind the GEMM the step up to the sums of u runs beside it
// (16 rows of 6144 outputs in three layers 16.9 -> 15.0 us, the 48 rows 27.6 -> 26.3; y and the sums' exchange behind one another instead, 15.8 and 26.7).
template <int R16>
struct Decode {
    static constexpr int kRows = 16, kRanks = 16 * R16, kCluster = 8;           // (most CTAs of a cluster)
    static constexpr int kBytes = (kWarps + kCluster) * kRows * kRanks * 4 + Operand<R16>::pieces(kRows) * 16 + kRows * 4 + kWarps * kRows * 4;
    static_assert(kBytes <= 227 * 1024, "shared memory of an SM");
};
// The lane's part of 32 columns of the second factor and of y, on its way: 16-byte pieces, or, where rows lie on no 16-byte boundary, the halves that it needs (shifting
// pieces into place takes more instructions than these loads)
template <int R16, bool VEC>
struct Columns {
    uint4 b[R16][4], y[2];
    // L and batch only for the checks; src: the lane's 8 columns of its first row; n of them are inside; ranks: of its rows 16 k + i those below this exist
    __device__ __forceinline__ void load(const DecodeLayer& L, int batch, const __half* src, int m_all, int n, int ranks, const __half* const (&y_src)[2], const bool (&has)[2], int n_y) {
#pragma unroll
        for (int k = 0; k < R16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) b[k][i] = 16 * k + i < ranks && n > 0 && RABIT_IN_RANGE(inside(src + (size_t)(16 * k + i) * m_all, 16, L.b, (size_t)L.count * L.rank * m_all * 2)) ? *reinterpret_cast<const uint4*>(src + (size_t)(16 * k + i) * m_all) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int h = 0; h < 2; ++h) y[h] = has[h] && n_y > 0 && RABIT_IN_RANGE(inside(y_src[h], 16, L.y, (size_t)batch * m_all * 2)) ? *reinterpret_cast<const uint4*>(y_src[h]) : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void factor(uint32_t (&f)[R16][1][4][2], int odd) const {
        const uint32_t pick = odd ? 0x7632u : 0x5410u;
#pragma unroll
        for (int k = 0; k < R16; ++k)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                f[k][0][0][p] = __byte_perm(b[k][2 * p].x, b[k][2 * p + 1].x, pick);
                f[k][0][1][p] = __byte_perm(b[k][2 * p].y, b[k][2 * p + 1].y, pick);
                f[k][0][2][p] = __byte_perm(b[k][2 * p].z, b[k][2 * p + 1].z, pick);
                f[k][0][3][p] = __byte_perm(b[k][2 * p].w, b[k][2 * p + 1].w, pick);
            }
    }
    __device__ __forceinline__ uint4 row(int h) const { return y[h]; }
};
template <int R16>
struct Columns<R16, false> {
    unsigned short b[R16][4][4], y[2][8];
    __device__ __forceinline__ void load(const DecodeLayer& L, int batch, const __half* src, int m_all, int n, int ranks, const __half* const (&y_src)[2], const bool (&has)[2], int n_y) {
        const int odd = (threadIdx.x >> 2) & 1;                                 // which column of a pair the lane's fragments hold
#pragma unroll
        for (int k = 0; k < R16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned short* row = reinterpret_cast<const unsigned short*>(src + (size_t)(16 * k + i) * m_all) + odd;
#pragma unroll
                for (int q = 0; q < 4; ++q) b[k][i][q] = 16 * k + i < ranks && 2 * q + odd < n && RABIT_IN_RANGE(inside(row + 2 * q, 2, L.b, (size_t)L.count * L.rank * m_all * 2)) ? row[2 * q] : (unsigned short)0;
            }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 8; ++q) y[h][q] = has[h] && q < n_y && RABIT_IN_RANGE(inside(y_src[h] + q, 2, L.y, (size_t)batch * m_all * 2)) ? reinterpret_cast<const unsigned short*>(y_src[h])[q] : (unsigned short)0;
    }
    __device__ __forceinline__ void factor(uint32_t (&f)[R16][1][4][2], int) const {
#pragma unroll
        for (int k = 0; k < R16; ++k)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int p = 0; p < 2; ++p) f[k][0][q][p] = b[k][2 * p][q] | (uint32_t)b[k][2 * p + 1][q] << 16;
    }
    __device__ __forceinline__ uint4 row(int h) const {
        return make_uint4(y[h][0] | (uint32_t)y[h][1] << 16, y[h][2] | (uint32_t)y[h][3] << 16, y[h][4] | (uint32_t)y[h][5] << 16, y[h][6] | (uint32_t)y[h][7] << 16);
    }
};
template <int R16, bool VEC>
__global__ void __launch_bounds__(kThreads, R16 == 1 ? 2 : 1) decode_kernel(const __grid_constant__ DecodeParams P) {
    using D = Decode<R16>;
    using O = Operand<R16>;
    constexpr int kRows = D::kRows, kRanks = D::kRanks, NR = 2 * R16;
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    extern __shared__ __align__(16) unsigned char decode_smem[];
    float* red = reinterpret_cast<float*>(decode_smem);                         // [kWarps][kRows][kRanks]: the warps' sums
    float* inbox = red + kWarps * kRows * kRanks;                               // [kCluster][kRows][kRanks]: the CTAs' sums
    uint4* us = reinterpret_cast<uint4*>(inbox + D::kCluster * kRows * kRanks); // u as operand, then its rows' factors
    float* backs = reinterpret_cast<float*>(us + O::pieces(kRows));
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, tq = lane & 3;
    int* rows = reinterpret_cast<int*>(backs + kRows) + warp * kRows;           // the rows at hand (-1: none), every warp for itself
    const DecodeLayer& L = P.layer[blockIdx.z];
    const int n = L.n, m_all = L.m, rank = L.rank, row0 = (int)(blockIdx.x / parts) * kWindow, batch = min(kWindow, P.batch - row0);   // rows of the window
    const int groups = (m_all + 31) / 32, step = parts * kWarps;                // of 32 columns
    const uint32_t before = (1u << lane) - 1u;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bool waited = P.beside == 0;                                                // (beside the layer everything is read from L2, as in narrow_kernel)
    if (waited) asm volatile("griddepcontrol.wait;" ::: "memory");

    // rows `lane` and 32 + `lane` of the window
    int id = lane < batch ? __ldcg(P.ids + row0 + lane) : -1, id1 = 32 + lane < batch ? __ldcg(P.ids + row0 + 32 + lane) : -1;
    if (id >= L.count) id = -1;
    if (id1 >= L.count) id1 = -1;
    uint32_t same = __match_any_sync(kAll, id), same1 = 0u;                     // rows of the same adapter: in the first 32, in the second
    bool leads = id >= 0 && (same & before) == 0u, leads1 = false;              // the adapter's first row
    uint32_t same_of1 = 0u, same1_of1 = 0u;
    if (batch > 32) {
        same1_of1 = __match_any_sync(kAll, id1);
        for (uint32_t each = __ballot_sync(kAll, id1 >= 0 && (same1_of1 & before) == 0u); each != 0u; each &= each - 1u) {   // the adapters among the second 32 rows
            const int who = __ffs(each) - 1, v = __shfl_sync(kAll, id1, who);
            const uint32_t there = __shfl_sync(kAll, same1_of1, who), here = __ballot_sync(kAll, id == v);
            if (id == v) same1 = there;
            if (id1 == v) same_of1 = here;
        }
        leads1 = id1 >= 0 && same_of1 == 0u && (same1_of1 & before) == 0u;
    }
    // items: 16 rows of an adapter each, in the order of the adapters' first rows
    int items = leads ? (__popc(same) + __popc(same1) + kRows - 1) / kRows : 0, items1 = leads1 ? (__popc(same1_of1) + kRows - 1) / kRows : 0;
    int end = items, end1 = items1;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(kAll, end, d), v1 = __shfl_up_sync(kAll, end1, d);
        if (lane >= d) { end += v; end1 += v1; }
    }
    const int total0 = __shfl_sync(kAll, end, 31), total = total0 + __shfl_sync(kAll, end1, 31);
    end1 += total0;
    if ((int)blockIdx.y < total) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (all CTAs of the cluster run before any writes to another's memory)
    for (int turn = blockIdx.y; turn < total; turn += (int)gridDim.y) {
        const uint32_t at = __ballot_sync(kAll, turn >= end - items && turn < end), at1 = __ballot_sync(kAll, turn >= end1 - items1 && turn < end1);
        const int who = __ffs(at ? at : at1) - 1;
        const int cur = __shfl_sync(kAll, at ? id : id1, who), skip = (turn - __shfl_sync(kAll, at ? end - items : end1 - items1, who)) * kRows;
        const uint32_t mask = __shfl_sync(kAll, at ? same : 0u, who), mask1 = __shfl_sync(kAll, at ? same1 : same1_of1, who);
        __syncwarp();
        if (lane < kRows) rows[lane] = -1;
        __syncwarp();
        const int place = __popc(mask & before) - skip, place1 = __popc(mask) + __popc(mask1 & before) - skip;
        if ((mask >> lane & 1u) && place >= 0 && place < kRows) rows[place] = row0 + lane;
        if ((mask1 >> lane & 1u) && place1 >= 0 && place1 < kRows) rows[place1] = row0 + 32 + lane;
        __syncwarp();
        const bool has[2] = {rows[gq] >= 0, rows[8 + gq] >= 0};
        const size_t row[2] = {(size_t)max(rows[gq], 0), (size_t)max(rows[8 + gq], 0)};
        const float scale = RABIT_IN_RANGE(who >= 0 && cur >= 0 && cur < L.count) ? __ldcg(L.scale + cur) : 0.f;

        float acc[NR][4] = {};
        {
            const int units = n / 32, worker = part * kWarps + warp, workers = parts * kWarps;
            const int u0 = (int)((long long)units * worker / workers), u1 = (int)((long long)units * (worker + 1) / workers);
            const __half* a = L.a + ((size_t)cur * rank + gq) * n + 8 * tq;
            const __half* x[2] = {L.x + row[0] * n + 8 * tq, L.x + row[1] * n + 8 * tq};
            struct Loads {
                uint4 x[2], a[NR];
            };
            auto load = [&](Loads& l, int u) {
                const bool in = u < u1;
                const size_t col = (size_t)u * 32;
#pragma unroll
                for (int m = 0; m < 2; ++m) l.x[m] = in && has[m] && RABIT_IN_RANGE(inside(x[m] + col, 16, L.x, (size_t)P.batch * n * 2)) ? __ldcg(reinterpret_cast<const uint4*>(x[m] + col)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int j = 0; j < NR; ++j) l.a[j] = in && 8 * j + gq < rank && RABIT_IN_RANGE(inside(a + (size_t)(8 * j) * n + col, 16, L.a, (size_t)L.count * rank * n * 2)) ? __ldcg(reinterpret_cast<const uint4*>(a + (size_t)(8 * j) * n + col)) : make_uint4(0u, 0u, 0u, 0u);
            };
            auto multiply = [&](const Loads& l) {
#pragma unroll
                for (int j = 0; j < NR; ++j) {
                    mma_f16(acc[j], l.x[0].x, l.x[1].x, l.x[0].y, l.x[1].y, l.a[j].x, l.a[j].y);
                    mma_f16(acc[j], l.x[0].z, l.x[1].z, l.x[0].w, l.x[1].w, l.a[j].z, l.a[j].w);
                }
            };
            float* own = red + ((size_t)warp * kRows + gq) * kRanks + 2 * tq;   // the lane's sums: rows gq and gq + 8, ranks 8 j + 2 tq and the next
            auto flush = [&](bool first) {                                  // (the tensor core truncates: chains of at most 16 MMAs)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < NR; ++j) {
                        float2* at = reinterpret_cast<float2*>(own + 8 * m * kRanks + 8 * j);
                        float2 v = make_float2(acc[j][2 * m], acc[j][2 * m + 1]);
                        if (!first) {
                            const float2 old = *at;
                            v.x += old.x;
                            v.y += old.y;
                        }
                        *at = v;
                        acc[j][2 * m] = acc[j][2 * m + 1] = 0.f;
                    }
            };
            Loads even, odd;
            load(even, u0);
            int pairs = 0;
#pragma unroll 1
            for (int u = u0; u < u1; u += 2) {
                load(odd, u + 1);
                multiply(even);
                load(even, u + 2);
                multiply(odd);
                if (++pairs % 4 == 0) flush(pairs == 4);
            }
            if (pairs % 4 != 0 || pairs == 0) flush(pairs < 4);
        }

        if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");         // y
        waited = true;
        // the second factor's entries and y of the warp's first 32 columns are on their way while u is put together
        const __half* b = L.b + ((size_t)cur * rank + 4 * tq) * m_all + 8 * (gq >> 1);
        __half* y[2] = {L.y + row[0] * m_all + 8 * tq, L.y + row[1] * m_all + 8 * tq};
        int g = warp * parts + part;                                        // neighbouring columns to different SMs
        constexpr int kSets = R16 <= (VEC ? 4 : 2) ? 2 : 1;                      // sets of 32 columns on their way
        Columns<R16, VEC> sets[kSets];
        auto load_columns = [&](Columns<R16, VEC>& l, int g) {
            const __half* const y_src[2] = {y[0] + 32 * g, y[1] + 32 * g};
            l.load(L, P.batch, b + 32 * g, m_all, g < groups ? m_all - 32 * g - 8 * (gq >> 1) : 0, rank - 4 * tq, y_src, has, g < groups ? m_all - 32 * g - 8 * tq : 0);
        };
#pragma unroll
        for (int q = 0; q < kSets; ++q) load_columns(sets[q], g + q * step);
        __syncthreads();
        cluster_wait();
        for (int e = threadIdx.x; e < kRows * kRanks / 4; e += kThreads) {
            float4 s = reinterpret_cast<const float4*>(red)[e];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) {
                const float4 v = reinterpret_cast<const float4*>(red)[w * (kRows * kRanks / 4) + e];
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
#pragma unroll 4
            for (int q = 0; q < D::kCluster; ++q)
                if (q < parts) reinterpret_cast<float4*>(cluster.map_shared_rank(inbox, q))[part * (kRows * kRanks / 4) + e] = s;
        }
        cluster.sync();
        for (int e = threadIdx.x; e < kRows * kRanks / 4; e += kThreads) {
            float4 s = reinterpret_cast<const float4*>(inbox)[e];
            for (int q = 1; q < parts; ++q) {
                const float4 v = reinterpret_cast<const float4*>(inbox)[q * (kRows * kRanks / 4) + e];
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            const int r = e / (kRanks / 4), j = e % (kRanks / 4) * 4;
            // (beyond the rank an infinite x has met zeros)
            s = make_float4(j < rank ? s.x : 0.f, j + 1 < rank ? s.y : 0.f, j + 2 < rank ? s.z : 0.f, j + 3 < rank ? s.w : 0.f);
            const float back = split_row<R16>(us, r, j / 4, s);
            if (j == 0) backs[r] = back;
            if (part == 0 && j < rank && rows[r] >= 0 && RABIT_IN_RANGE(rows[r] < P.batch)) store_4(L.u + (size_t)rows[r] * rank + j, s, rank - j, rank % 4 == 0);
        }
        __syncthreads();
        if (turn + (int)gridDim.y < total) cluster_arrive();                // the inbox has been read: sums of the next item may come

        auto widen_columns = [&](Columns<R16, VEC>& l, int g) {
            if (g >= groups) return;
            uint32_t f[R16][1][4][2];
            l.factor(f, gq & 1);
            const uint4 old[2] = {l.row(0), l.row(1)};
            load_columns(l, g + kSets * step);
            float sum[1][4][4];
#pragma unroll
            for (int k = 0; k < R16; ++k) widen_step<1>(sum, k == 0, us + O::at(gq) + 4 * k + tq, O::kSecond, f[k]);
            const int left_cols = m_all - 32 * g - 8 * tq;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (has[h] && left_cols > 0 && RABIT_IN_RANGE(inside(y[h] + 32 * g, 2 * min(left_cols, 8), L.y, (size_t)P.batch * m_all * 2))) widen_store<VEC>(y[h] + 32 * g, left_cols, old[h], sum[0], h, scale * backs[8 * h + gq]);
        };
        for (; g < groups; g += kSets * step) {
#pragma unroll
            for (int q = 0; q < kSets; ++q) widen_columns(sets[q], g + q * step);
        }
    }
    if (!waited && blockIdx.y == 0) asm volatile("griddepcontrol.wait;" ::: "memory");   // (no item at all: the grid ends behind the layer's even so)
    if (blockIdx.y == 0 && part == 0) {                                         // rows without adapter: u is zero
        uint32_t bare[2] = {__ballot_sync(kAll, id < 0 && lane < batch), __ballot_sync(kAll, id1 < 0 && 32 + lane < batch)};
        int turn = 0;
        for (int h = 0; h < 2; ++h)
            for (; bare[h] != 0u; bare[h] &= bare[h] - 1u)
                if (turn++ % kWarps == warp)
                    for (int j = lane; j < rank && RABIT_IN_RANGE(row0 + 32 * h + __ffs(bare[h]) - 1 < P.batch); j += 32) L.u[(size_t)(row0 + 32 * h + __ffs(bare[h]) - 1) * rank + j] = 0.f;
    }
}

// ---- out[i][j][d] (+)= scale[i] * sum over the adapter's rows of low[t][j] v[t][d] -----------------------------

struct FactorSide {
    const __half* v;
    const float* low;
    float* out;
    int side, blocks;                                                           // column blocks of this side
};
struct FactorParams {
    FactorSide s[2];
    const int* ids;
    const float* scale;
    int batch, rank, accumulate;
};
constexpr int kFactorThreads = 512, kFactorWarps = kFactorThreads / 32, kFactorList = 1024, kFactorChunk = 64;

template <int GROUPS>
struct Factor {                                                                 // GROUPS warps side by side for the ranks, kColWarps for the columns, kSlices for the rows of a tile
    static constexpr int kRanks = 16 * GROUPS, kRows = GROUPS == 8 ? 32 : 64, kColWarps = GROUPS == 8 ? 2 : 4, kSlices = kFactorWarps / (GROUPS * kColWarps);
    static constexpr int kCols = 64 * kColWarps, kSteps = kRows / 16 / kSlices; // MMAs of 16 rows of a warp in a tile
    static constexpr int kVStride = kCols * 2 + 16, kLowStride = kRanks + 4, kAStride = kRows * 2 + 16;         // bytes, words, bytes: rows that are read together meet in few banks
    static constexpr int kVBytes = kRows * kVStride, kStageBytes = kVBytes + kRows * kLowStride * 4;
    static constexpr int kStages = GROUPS == 8 ? 4 : 3, kABytes = kRanks * kAStride;
    static constexpr int kAAt = kStages * kStageBytes, kBackAt = kAAt + 4 * kABytes, kListAt = kBackAt + 2 * kRanks * 4, kBytes = kListAt + kFactorList * 4;
    static_assert(kSteps >= 1 && kSlices * kRanks * kCols * 4 <= kBytes && kBytes <= 226 * 1024, "the sums fit, one CTA per SM");
};
__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_trans(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// Ranks by columns as m16n8k16 MMAs over the rows, v as it is, low as two fp16 parts of a power of two per rank and tile of 64 rows (v and low meet as matrices
// with the rows inside, so low is turned when it is split).  A warp takes 16 ranks and 64 columns, GROUPS warps the same columns; 16 warps, because what a
// tile costs beside its MMAs (copies, splitting, barriers) is then shared by 256 columns.  The rows of a
// cluster's adapter are dealt out to its CTAs in chunks of 64; a CTA first lists the rows that are its adapter's, so other rows are neither read nor
// multiplied by zero (0 * NaN), then streams them through a ring of stages; the next tile is split
// beside the MMAs of the one at hand, half of the warps doing the one first, half the other.
// Sums of a tile are added up in fp32 registers (the tensor core truncates), the CTAs' sums over the cluster in order.
// Bound: 2048 rows of 4096 and 4096 columns, rank 16: 15.5 us (33.5 MB: 5.1; per tile of 64 rows 920 clocks are copies, 640 splitting, 410 MMAs, and a CTA's start and
// the sum over the cluster cost as much as eight tiles); 4096 rows of 11008 and 4096 columns, two adapters of rank 64: 98 us (124 MB: 19; MMAs 29), issue slots.
template <int GROUPS, bool VEC>
__global__ void __launch_bounds__(kFactorThreads, 1) factor_kernel(const __grid_constant__ FactorParams P) {
    using F = Factor<GROUPS>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int counts[kFactorWarps], found;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, tq = lane & 3;
    const int group = warp % GROUPS, wc = warp / GROUPS % F::kColWarps, slice = warp / (GROUPS * F::kColWarps);
    int block = (int)blockIdx.x / parts;
    const FactorSide& S = P.s[block < P.s[0].blocks ? 0 : 1];
    if (block >= P.s[0].blocks) block -= P.s[0].blocks;
    const int adapter = blockIdx.y, side = S.side, first = block * F::kCols, rank = P.rank;
    const bool fours = rank % 4 == 0;
    int* list = reinterpret_cast<int*>(smem + F::kListAt);
    float* backs = reinterpret_cast<float*>(smem + F::kBackAt);                 // [2][kRanks]
    const uint32_t smem32 = (uint32_t)__cvta_generic_to_shared(smem);
    // the lane's row of the 8 x 8 matrices that it names: of v rows of the tile by columns, of low ranks by rows of the tile
    const uint32_t v_at = smem32 + (uint32_t)((lane & 15) * F::kVStride + (wc * 64 + (lane >> 4) * 8) * 2);
    const uint32_t a_at = smem32 + (uint32_t)(F::kAAt + (group * 16 + (lane & 15)) * F::kAStride + (lane >> 4) * 16);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const bool prepare_first = (warp & 4) != 0;                                 // half of a scheduler's warps copy and split while the others multiply
    float sum[8][4] = {};
    int n_rows = 0;                                                             // of the adapter, among the CTA's
    for (long long base = 0; base < P.batch; base += (long long)kFactorList * parts) {
        // the rows of this round that are the adapter's, in order
        int n_list = 0;
        for (int at = 0; at < kFactorList; at += kFactorThreads) {
            const int pos = at + (int)threadIdx.x;
            const long long t = base + ((long long)(pos / kFactorChunk) * parts + part) * kFactorChunk + pos % kFactorChunk;
            if (base + (long long)(at / kFactorChunk) * parts * kFactorChunk >= P.batch) break;
            const bool hit = t < P.batch && P.ids[t] == adapter;
            const uint32_t hits = __ballot_sync(0xFFFFFFFFu, hit);
            if (lane == 0) counts[warp] = __popc(hits);
            __syncthreads();
            int before = n_list;
            for (int w = 0; w < kFactorWarps; ++w) {
                if (w < warp) before += counts[w];
                n_list += counts[w];
            }
            if (hit && RABIT_IN_RANGE(before + __popc(hits & ((1u << lane) - 1u)) < kFactorList)) list[before + __popc(hits & ((1u << lane) - 1u))] = (int)t;
            __syncthreads();
        }
        n_rows += n_list;
        const int n_tiles = (n_list + F::kRows - 1) / F::kRows;
        auto fetch = [&](int tile) {
            unsigned char* stage = smem + tile % F::kStages * F::kStageBytes;
            if (tile < n_tiles) {
                constexpr int kPieces = F::kCols / 8;                           // 16 bytes of a row each
#pragma unroll
                for (int i0 = 0; i0 < F::kRows * kPieces; i0 += kFactorThreads) {
                    const int i = i0 + (int)threadIdx.x, r = i / kPieces, col = first + i % kPieces * 8, at = tile * F::kRows + r;
                    const bool in = at < n_list && col < side;
                    const __half* src = in ? S.v + (size_t)list[at] * side + col : S.v;
                    unsigned char* dst = stage + r * F::kVStride + i % kPieces * 16;
                    if (!RABIT_IN_RANGE(inside(dst, 16, stage, F::kVBytes) && (!in || inside(src, 2 * min(side - col, 8), S.v, (size_t)P.batch * side * 2)))) continue;
                    if (VEC) copy_async_16(dst, src, in);
                    else *reinterpret_cast<uint4*>(dst) = load_8(src, in ? side - col : 0, S.v, S.v + (size_t)P.batch * side);
                }
                float* low = reinterpret_cast<float*>(stage + F::kVBytes);
                constexpr int kFours = F::kRanks / 4;
                for (int i = threadIdx.x; i < F::kRows * kFours; i += kFactorThreads) {
                    const int r = i / kFours, j = i % kFours * 4, at = tile * F::kRows + r;
                    const bool in = at < n_list;
                    const float* src = in ? S.low + (size_t)list[at] * rank + j : S.low;
                    float* dst = low + r * F::kLowStride + j;
                    if (!RABIT_IN_RANGE(inside(dst, 16, stage + F::kVBytes, F::kRows * F::kLowStride * 4) && (!in || j >= rank || inside(src, 4 * min(rank - j, 4), S.low, (size_t)P.batch * rank * 4)))) continue;
                    if (fours) {
                        copy_async_16(dst, in && j < rank ? src : S.low, in && j < rank);
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) copy_async_4(dst + q, in && j + q < rank ? src + q : S.low, in && j + q < rank);
                    }
                }
            }
            copy_async_commit();
        };
        // low of a tile as operand: neighbouring lanes share a rank's rows
        auto split = [&](int tile) {
            if (tile >= n_tiles) return;
            constexpr int kShare = kFactorThreads / F::kRanks, kEach = F::kRows / kShare;
            const float* low = reinterpret_cast<const float*>(smem + tile % F::kStages * F::kStageBytes + F::kVBytes);
            const int j = threadIdx.x / kShare, sub = threadIdx.x % kShare;
            float v[kEach], largest = 0.f;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                v[i] = low[(sub + kShare * i) * F::kLowStride + j];
                largest = fmaxf(largest, finite_size(v[i]));
            }
#pragma unroll
            for (int d = 1; d < kShare; d <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, d));
            float to, back;
            range_of(largest, to, back);
            if (sub == 0) backs[(tile & 1) * F::kRanks + j] = back;
            __half* out = reinterpret_cast<__half*>(smem + F::kAAt + (tile & 1) * 2 * F::kABytes + j * F::kAStride) + sub;
#pragma unroll
            for (int i = 0; i < kEach; ++i) split_f16(v[i], to, out[kShare * i], out[F::kABytes / 2 + kShare * i]);
        };
#pragma unroll
        for (int tile = 0; tile < F::kStages - 1; ++tile) fetch(tile);
        copy_async_wait<F::kStages - 2>();
        __syncthreads();
        split(0);
        for (int tile = 0; tile < n_tiles; ++tile) {
            copy_async_wait<F::kStages - 3>();
            __syncthreads();                                                    // the next tile is there, this one is split, and the slots of the one before are free
            auto prepare = [&]() {
                fetch(tile + F::kStages - 1);
                split(tile + 1);
            };
            if (prepare_first) prepare();
            const uint32_t v = v_at + (uint32_t)(tile % F::kStages * F::kStageBytes), a = a_at + (uint32_t)((tile & 1) * 2 * F::kABytes);
            float acc[8][4];
#pragma unroll
            for (int s0 = 0; s0 < F::kSteps; ++s0) {
                const int s = slice * F::kSteps + s0;                           // 16 rows of the tile
                uint32_t hi[4], lo[4], b[4][4];
                ldmatrix(hi, a + (uint32_t)(s * 32));
#pragma unroll
                for (int q = 0; q < 4; ++q) ldmatrix_trans(b[q], v + (uint32_t)(s * 16 * F::kVStride + q * 32));
                ldmatrix(lo, a + (uint32_t)(F::kABytes + s * 32));
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    if (s0 == 0) mma_f16_first(acc[q], hi[0], hi[1], hi[2], hi[3], b[q >> 1][2 * (q & 1)], b[q >> 1][2 * (q & 1) + 1]);
                    else mma_f16(acc[q], hi[0], hi[1], hi[2], hi[3], b[q >> 1][2 * (q & 1)], b[q >> 1][2 * (q & 1) + 1]);
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) mma_f16(acc[q], lo[0], lo[1], lo[2], lo[3], b[q >> 1][2 * (q & 1)], b[q >> 1][2 * (q & 1) + 1]);
            }
            const float back0 = backs[(tile & 1) * F::kRanks + group * 16 + gq], back1 = backs[(tile & 1) * F::kRanks + group * 16 + 8 + gq];
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[q][e] = fmaf(e < 2 ? back0 : back1, acc[q][e], sum[q][e]);
            if (!prepare_first) prepare();
        }
        copy_async_wait<0>();
        __syncthreads();                                                        // (the list is written again)
    }
    // the CTA's sums [slice][rank][column of the block], then over the cluster
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int e = 0; e < 4; e += 2)
            *reinterpret_cast<float2*>(sums + (slice * F::kRanks + group * 16 + gq + 4 * e) * F::kCols + wc * 64 + 8 * q + 2 * tq) = make_float2(sum[q][e], sum[q][e + 1]);
    if (F::kSlices > 1) {
        __syncthreads();
        float4* fours_of = reinterpret_cast<float4*>(sums);
        for (int e = threadIdx.x; e < F::kRanks * F::kCols / 4; e += kFactorThreads) {
            float4 total = fours_of[e];
#pragma unroll
            for (int q = 1; q < F::kSlices; ++q) {
                const float4 v = fours_of[q * (F::kRanks * F::kCols / 4) + e];
                total.x += v.x; total.y += v.y; total.z += v.z; total.w += v.w;
            }
            fours_of[e] = total;
        }
    }
    if (threadIdx.x == 0) found = n_rows;
    float scale = P.scale[adapter];
    cluster.sync();
    // An adapter that no row names has the gradient zero whatever its scale is: its slot in the pool may never have been written.  Its sums are zero, so that matters (0 * NaN)
    // where the scale is not finite; asking the cluster for the rows each time took 0.3 to 1.2 us.
    if (!(fabsf(scale) <= 3.402823466e38f)) {
        int named = 0;
        for (int q = 0; q < parts; ++q) named |= *cluster.map_shared_rank(&found, q);
        if (named == 0) scale = 0.f;
    }
    const int cols = min(F::kCols, side - first);
    const bool side_fours = side % 4 == 0;
    for (int e = part * kFactorThreads + threadIdx.x; e < rank * F::kCols / 4; e += parts * kFactorThreads) {
        const int j = e / (F::kCols / 4), c = e % (F::kCols / 4) * 4;
        if (c >= cols) continue;
        float4 total = cluster_sum(cluster, sums, parts, e);
        total.x *= scale; total.y *= scale; total.z *= scale; total.w *= scale;
        float* at = S.out + ((size_t)adapter * rank + j) * side + first + c;
        if (!RABIT_IN_RANGE(inside(at, 4 * min(cols - c, 4), S.out, (size_t)gridDim.y * rank * side * 4))) continue;
        if (P.accumulate) {
            if (side_fours) {
                const float4 old = *reinterpret_cast<const float4*>(at);
                total.x += old.x; total.y += old.y; total.z += old.z; total.w += old.w;
            } else {
                total.x += at[0];
                if (c + 1 < cols) total.y += at[1];
                if (c + 2 < cols) total.z += at[2];
                if (c + 3 < cols) total.w += at[3];
            }
        }
        store_4(at, total, cols - c, side_fours);
    }
    cluster.sync();
}

// ---- launches ----------------------------------------------------------------------------------------------

template <typename Params>
cudaError_t launch(void (*kernel)(Params), dim3 grid, int cluster, int smem, const Params& P, cudaStream_t stream, int threads = kThreads) {
    if (smem > 48 * 1024) {                                                     // (an attribute of the function on the current device; setting it again is cheap)
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    if (cluster > 0) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim = {(unsigned)cluster, 1, 1};
        ++cfg.numAttrs;
    }
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
    return cudaLaunchKernelEx(&cfg, kernel, P);
}

// Clusters that share the adapters of a tile of rows: more while there are few tiles.
int shares_for(int batch) { return batch < 2048 ? 4 : 2; }

cudaError_t launch_narrow(NarrowParams& P, int n_layers, int max_rank, cudaStream_t stream) {
    const int wm = P.batch * (long long)n_layers <= 512 ? 2 : P.batch < 2048 ? 4 : 8;   // 32, 64 or 128 rows to a tile
    const long long tiles = (P.batch + 16 * wm - 1) / (16 * wm);
    P.shares = shares_for(P.batch);
    int c = kMaxCluster;
    while (c > 1 && tiles * n_layers * c > 400) c /= 2;
    const dim3 grid((unsigned)(tiles * c), (unsigned)P.shares, (unsigned)n_layers);
    auto go = [&](auto kernel, int bytes) { return launch(kernel, grid, c, bytes, P, stream); };
    if (wm == 2)
        return max_rank <= 16 ? go(narrow_kernel<2, 2>, Narrow<2, 2>::kBytes) : max_rank <= 32 ? go(narrow_kernel<4, 2>, Narrow<4, 2>::kBytes)
             : max_rank <= 64 ? go(narrow_kernel<8, 2>, Narrow<8, 2>::kBytes) : go(narrow_kernel<16, 2>, Narrow<16, 2>::kBytes);
    if (wm == 4)
        return max_rank <= 16 ? go(narrow_kernel<2, 4>, Narrow<2, 4>::kBytes) : max_rank <= 32 ? go(narrow_kernel<4, 4>, Narrow<4, 4>::kBytes)
             : max_rank <= 64 ? go(narrow_kernel<8, 4>, Narrow<8, 4>::kBytes) : go(narrow_kernel<16, 4>, Narrow<16, 4>::kBytes);
    return max_rank <= 16 ? go(narrow_kernel<2, 8>, Narrow<2, 8>::kBytes) : max_rank <= 32 ? go(narrow_kernel<4, 8>, Narrow<4, 8>::kBytes)
         : max_rank <= 64 ? go(narrow_kernel<8, 8>, Narrow<8, 8>::kBytes) : go(narrow_kernel<16, 8>, Narrow<16, 8>::kBytes);
}

template <int R16, bool VEC>
cudaError_t launch_widen(WidenParams& P, int n_layers, int max_m, cudaStream_t stream) {
    // as many row blocks to a CTA as leave two CTAs for every SM (296; one more would be a second wave)
    using W = Widen<R16, VEC>;
    const long long cols = (max_m + W::kCols - 1) / W::kCols, row_blocks = (P.batch + kWidenRows - 1) / kWidenRows;
    const long long along = std::min(std::max(296 / (cols * n_layers), 1LL), 65535LL);
    P.blocks = (int)((row_blocks + along - 1) / along);
    const dim3 grid((unsigned)cols, (unsigned)((row_blocks + P.blocks - 1) / P.blocks), (unsigned)n_layers);
    return launch(widen_kernel<R16, VEC>, grid, 0, W::kBytes, P, stream);
}

template <int R16, bool VEC>
cudaError_t launch_decode(const DecodeParams& P, int n_layers, int max_count, cudaStream_t stream) {
    // a window has an item for every adapter that its rows can name, and one for every 16 rows beyond that; where there are several windows, CTAs for the first 12 (the
    // others come in turn).  Clusters as large as leave the CTAs of one wave; those without an item end at once.
    const int windows = (P.batch + kWindow - 1) / kWindow, all = std::min(std::min(P.batch, kWindow), max_count) + std::min(P.batch, kWindow) / 16, items = windows == 1 ? all : std::min(all, 12);
    int c = Decode<R16>::kCluster;
    while (c > 2 && (long long)windows * items * n_layers * c > (R16 == 1 ? 296 : 222)) c /= 2;
    return launch(decode_kernel<R16, VEC>, dim3((unsigned)(windows * c), (unsigned)items, (unsigned)n_layers), c, Decode<R16>::kBytes, P, stream);
}

template <int GROUPS>
cudaError_t launch_factor(FactorParams& P, int count, cudaStream_t stream) {
    using F = Factor<GROUPS>;
    for (FactorSide& s : P.s) s.blocks = (s.side + F::kCols - 1) / F::kCols;
    const bool vec = P.s[0].side % 8 == 0 && P.s[1].side % 8 == 0;
    const long long blocks = (long long)P.s[0].blocks + P.s[1].blocks;
    // the cluster whose waves of one CTA per SM take least; what a CTA does before and after its tiles takes as long as about five of them
    const long long tiles = (P.batch + F::kRows - 1) / F::kRows;
    int c = 1;
    double least = 1e300;
    for (int q = 1; q <= 8 && q <= tiles; ++q) {
        const double cost = (double)((blocks * count * q + 147) / 148) * (5.0 + (double)((tiles + q - 1) / q) / count);
        if (cost < least) { least = cost; c = q; }
    }
    const dim3 grid((unsigned)(blocks * c), (unsigned)count);
    return vec ? launch(factor_kernel<GROUPS, true>, grid, c, F::kBytes, P, stream, kFactorThreads) : launch(factor_kernel<GROUPS, false>, grid, c, F::kBytes, P, stream, kFactorThreads);
}

int check_pool(const char* who, const rabit_adapters* A) {
    if (!A->a || !A->b || !A->scale) return rabit_fail(RABIT_INVALID_ARG, "%s: null pointer in the adapters", who);
    if (A->count < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: count must be >= 1 (got %d)", who, A->count);
    if (A->rank < 1 || A->rank > RABIT_MAX_RANK) return rabit_fail(RABIT_UNSUPPORTED_SHAPE, "%s: rank must be 1..%d (got %d)", who, RABIT_MAX_RANK, A->rank);
    if (A->n_in < 1 || A->n_out < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: n_in and n_out must be positive (got %d, %d)", who, A->n_in, A->n_out);
    if ((((uintptr_t)A->a) & 15u) || (((uintptr_t)A->b) & 15u) || (((uintptr_t)A->scale) & 3u))
        return rabit_fail(RABIT_INVALID_ARG, "%s: factors must be 16-byte aligned, scale 4-byte aligned", who);
    return RABIT_OK;
}

struct Range {
    const void* p;
    size_t bytes;
    bool meets(const Range& o) const { return p && o.p && rabit_ranges_overlap(p, bytes, o.p, o.bytes); }
};

// What rabit_linear and rabit_linear_group check of these arguments, before the first kernel of an adapted call is enqueued.
int check_layers(const char* who, const rabit_layer* const* layers, const void* const* xs, void* const* ys, int n_layers, int batch) {
    for (int l = 0; l < n_layers; ++l) {
        if ((((uintptr_t)xs[l]) & 15u) || (((uintptr_t)ys[l]) & 15u)) return rabit_fail(RABIT_INVALID_ARG, "%s: x and y must be 16-byte aligned (entry %d)", who, l);
        if (layers[l]->device != layers[0]->device) return rabit_fail(RABIT_INVALID_ARG, "%s: entry %d lives on another device", who, l);
        const Range r_y{ys[l], (size_t)batch * layers[l]->geom.M * 2};
        for (int m = 0; m < n_layers; ++m) {
            if (r_y.meets(Range{xs[m], (size_t)batch * layers[m]->geom.N * 2})) return rabit_fail(RABIT_INVALID_ARG, "%s: output %d overlaps input %d", who, l, m);
            if (m > l && r_y.meets(Range{ys[m], (size_t)batch * layers[m]->geom.M * 2})) return rabit_fail(RABIT_INVALID_ARG, "%s: outputs %d and %d overlap", who, l, m);
        }
    }
    return RABIT_OK;
}

int adapted_call(const char* who, const rabit_layer* const* layers, const rabit_adapters* const* adapters, const void* const* xs, const int* ids,
                 void* const* ys, float* const* us, int n_layers, int batch, void* stream) {
    rabit_clear_error();
    if (!layers || !adapters || !xs || !ys || !us) return rabit_fail(RABIT_INVALID_ARG, "%s: null array", who);
    if (n_layers < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: n_layers must be >= 1 (got %d)", who, n_layers);
    if (batch < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: batch must be >= 1 (got %d)", who, batch);
    if (batch > kMostRows) return rabit_fail(RABIT_UNSUPPORTED_SHAPE, "%s: batch must be <= %d (got %d)", who, kMostRows, batch);
    if (!ids || (((uintptr_t)ids) & 3u)) return rabit_fail(RABIT_INVALID_ARG, "%s: ids is NULL or misaligned", who);
    const Range r_ids{ids, (size_t)batch * 4};
    for (int l = 0; l < n_layers; ++l) {
        if (!layers[l] || !xs[l] || !ys[l]) return rabit_fail(RABIT_INVALID_ARG, "%s: null layer, x or y (entry %d)", who, l);
        const RabitGeom& G = layers[l]->geom;
        const Range r_y{ys[l], (size_t)batch * G.M * 2};
        if (r_y.meets(r_ids)) return rabit_fail(RABIT_INVALID_ARG, "%s: y overlaps ids (entry %d)", who, l);
        const rabit_adapters* A = adapters[l];
        if (!A) continue;
        int rc = check_pool(who, A);
        if (rc != RABIT_OK) return rc;
        if (A->n_in != G.N || A->n_out != G.M)
            return rabit_fail(RABIT_INVALID_ARG, "%s: adapters of %d -> %d beside a layer of %d -> %d (entry %d)", who, A->n_in, A->n_out, G.N, G.M, l);
        if (!us[l] || (((uintptr_t)us[l]) & 15u)) return rabit_fail(RABIT_INVALID_ARG, "%s: u is NULL or not 16-byte aligned (entry %d)", who, l);
        const Range r_u{us[l], (size_t)batch * A->rank * 4};
        if (r_u.meets(r_ids)) return rabit_fail(RABIT_INVALID_ARG, "%s: u overlaps ids (entry %d)", who, l);
        for (int m = 0; m < n_layers; ++m) {                     // (what y may not overlap besides: rabit_linear and rabit_linear_group)
            const rabit_adapters* O = adapters[m];
            if (layers[m] && xs[m] && ys[m] && (r_u.meets(Range{xs[m], (size_t)batch * layers[m]->geom.N * 2}) || r_u.meets(Range{ys[m], (size_t)batch * layers[m]->geom.M * 2})))
                return rabit_fail(RABIT_INVALID_ARG, "%s: u overlaps x or y (entries %d, %d)", who, l, m);
            if (!O) continue;
            if (m != l && us[m] && r_u.meets(Range{us[m], (size_t)batch * O->rank * 4})) return rabit_fail(RABIT_INVALID_ARG, "%s: u of entries %d and %d overlap", who, l, m);
        }
        const Range factors[3] = {{A->a, (size_t)A->count * A->rank * A->n_in * 2}, {A->b, (size_t)A->count * A->rank * A->n_out * 2}, {A->scale, (size_t)A->count * 4}};
        for (const Range& f : factors)
            for (int m = 0; m < n_layers; ++m)
                if (layers[m] && ((ys[m] && f.meets(Range{ys[m], (size_t)batch * layers[m]->geom.M * 2})) || (adapters[m] && us[m] && f.meets(Range{us[m], (size_t)batch * adapters[m]->rank * 4}))))
                    return rabit_fail(RABIT_INVALID_ARG, "%s: y or u of entry %d overlaps the adapters of entry %d", who, m, l);
    }
    cudaStream_t st = (cudaStream_t)stream;
    int dev = -1;
    RABIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev != layers[0]->device) return rabit_fail(RABIT_INVALID_ARG, "%s: the layers live on device %d but device %d is current", who, layers[0]->device, dev);

    // The layers, u of all adapted ones beside or behind the last kernel of that, then the adapters' part on top of the outputs.  What the layers' calls refuse is
    // refused before anything of this call has run.
    int at[kMaxGroup], n = 0;
    auto each_group = [&](auto&& body) {
        cudaError_t e = cudaSuccess;
        n = 0;
        for (int l = 0; l < n_layers && e == cudaSuccess; ++l) {
            if (adapters[l]) at[n++] = l;
            if (n == kMaxGroup || (l == n_layers - 1 && n > 0)) {
                e = body();
                n = 0;
            }
        }
        return e;
    };
    if (int rc = check_layers(who, layers, xs, ys, n_layers, batch)) return rc;
    for (int l = 0; l < n_layers; ++l)
        if (int rc = rabit_check_call(*layers[l], batch)) return rc;
    // One launch behind the layer, or two?  The one reads the second factor again for every 16 rows, so rows times outputs decide; the two multiply every tile with
    // each adapter in it, so where the pool has many to name the one is taken further.  (B200, us with the layer, graph replays with 14 layers in turn, one launch / two.
    // Three adapters in prompts, rank 16: 200 rows of 4096 x 4096 22.8 / 23.5, 256 rows 25.3 / 26.5, 512 rows 36.4 / 36.7, 1000 rows of 1024 x 4096 28.0 / 28.8, 130 rows of 8192 x
    // 4096 29.9 / 28.2; rank 32: 256 rows of 4096 x 4096 28.5 / 29.3, 512 rows 38.2 / 36.7; rank 64: 130 rows 25.0 / 29.3, 200 rows 31.2 / 29.6; rank 128: 130 rows 34.9 / 35.9, 200 rows
    // 45.3 / 36.7.  Outputs that are not 16-byte pieces, 4099 x 4096: rank 16 80 rows 21.2 / 21.7, 90 rows 21.6 / 21.1, 130 rows 25.1 / 24.2; rank 32 256 rows 32.4 / 33.9;
    // rank 64 256 rows 38.2 / 44.4, 400 rows 48.3 / 47.7; rank 128 256 rows 54.6 / 58.3.  30 adapters among single tokens: rank 16 130 rows of 4096 x 4096 30 / 50, 512 rows 55 / 85; rank 64 512 rows 111 / 141.)
    // The ids are on the device, so the size of the pool stands for how many adapters the rows name.  Rows that name one of a pool of 32 lose by that: 512 rows of 4096 x
    // 4096 40.0 / 34.0 at rank 16, 47.7 / 38.9 at rank 64.  Up to 64 rows it is one launch whatever the rest: with 30 adapters 64 rows of 14336 x 4096 30 / 54 at rank 16,
    // 57 / 93 at rank 64, with eight 26.3 / 34.7 and 39.9 / 51.2; with three it loses where outputs are many, 26.5 / 22.8 and 35.9 / 27.4.
    bool vec = true;
    long long outputs = 0;
    int most_rank = 0, most_count = 0;
    for (int l = 0; l < n_layers; ++l) {
        if (!adapters[l]) continue;
        vec = vec && adapters[l]->n_out % 8 == 0;
        outputs += adapters[l]->n_out;
        most_rank = std::max(most_rank, adapters[l]->rank);
        most_count = std::max(most_count, adapters[l]->count);
    }
    const long long most = most_count > 8 ? 1LL << 21 : !vec && most_rank <= 16 ? 3LL << 17 : most_rank > 32 && vec ? 5LL << 17 : 1LL << 20;
    const bool decode = batch <= kWindow || (batch <= kDecodeRows && batch * outputs <= most);
    bool beside = false;
    if (int rc = rabit_run_layers(layers, xs, ys, n_layers, batch, stream, &beside)) return rc;
    // Beside the layer's last kernel where that one lets the next start late (the GEMM): what is before the layer is complete then, x, ids and the readers of u among
    // it, and u is made on the SMs that the GEMM leaves idle or leaves first (B200, layer and adapters, us, u before it / beside it: 300 rows of 1024 x 4096 rank
    // 16 21.9 / 19.5, 1200 rows of 11008 x 4096 rank 128 242 / 236, 4096 rows of 11008 x 4096 rank 16 633 / 626).  Behind another kernel u waits for it.
    cudaError_t e = cudaSuccess;
    if (!decode) {
        e = each_group([&] {
            NarrowParams P{};
            P.ids = ids;
            P.batch = batch;
            P.beside = beside;
            int max_rank = 0;
            for (int i = 0; i < n; ++i) {
                const rabit_adapters* A = adapters[at[i]];
                P.layer[i] = NarrowLayer{(const __half*)xs[at[i]], (const __half*)A->a, us[at[i]], A->n_in, A->rank, A->count};
                max_rank = std::max(max_rank, A->rank);
            }
            return launch_narrow(P, n, max_rank, st);
        });
        if (e != cudaSuccess) return rabit_fail(RABIT_CUDA_ERROR, "%s: launch failed: %s", who, cudaGetErrorString(e));
    }
    e = each_group([&] {
        DecodeParams D{};
        WidenParams P{};
        P.ids = D.ids = ids;
        P.batch = D.batch = batch;
        P.beside = D.beside = beside;
        int max_rank = 0, max_m = 0, max_count = 0;
        for (int i = 0; i < n; ++i) {
            const rabit_adapters* A = adapters[at[i]];
            P.layer[i] = WidenLayer{(const __half*)A->b, us[at[i]], A->scale, (__half*)ys[at[i]], A->n_out, A->rank, A->count};
            D.layer[i] = DecodeLayer{(const __half*)xs[at[i]], (const __half*)A->a, (const __half*)A->b, A->scale, us[at[i]], (__half*)ys[at[i]], A->n_in, A->n_out, A->rank, A->count};
            max_rank = std::max(max_rank, A->rank);
            max_m = std::max(max_m, A->n_out);
            max_count = std::max(max_count, A->count);
        }
        if (decode && vec) return max_rank <= 16 ? launch_decode<1, true>(D, n, max_count, st) : max_rank <= 32 ? launch_decode<2, true>(D, n, max_count, st)
                                : max_rank <= 64 ? launch_decode<4, true>(D, n, max_count, st) : launch_decode<8, true>(D, n, max_count, st);
        if (decode) return max_rank <= 16 ? launch_decode<1, false>(D, n, max_count, st) : max_rank <= 32 ? launch_decode<2, false>(D, n, max_count, st)
                         : max_rank <= 64 ? launch_decode<4, false>(D, n, max_count, st) : launch_decode<8, false>(D, n, max_count, st);
        if (vec) return max_rank <= 16 ? launch_widen<1, true>(P, n, max_m, st) : max_rank <= 32 ? launch_widen<2, true>(P, n, max_m, st)
                      : max_rank <= 64 ? launch_widen<4, true>(P, n, max_m, st) : launch_widen<8, true>(P, n, max_m, st);
        return max_rank <= 16 ? launch_widen<1, false>(P, n, max_m, st) : max_rank <= 32 ? launch_widen<2, false>(P, n, max_m, st)
             : max_rank <= 64 ? launch_widen<4, false>(P, n, max_m, st) : launch_widen<8, false>(P, n, max_m, st);
    });
    if (e != cudaSuccess) return rabit_fail(RABIT_CUDA_ERROR, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return RABIT_OK;
}

int gradients_call(const rabit_adapters* A, const void* x, const float* u, const void* dy, const float* p, const int* ids, float* da, float* db, int batch,
                   int accumulate, void* stream) {
    const char* who = "rabit_adapter_gradients";
    rabit_clear_error();
    if (!A || !x || !u || !dy || !p || !ids || !da || !db) return rabit_fail(RABIT_INVALID_ARG, "%s: null pointer", who);
    int rc = check_pool(who, A);
    if (rc != RABIT_OK) return rc;
    if (batch < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: batch must be >= 1 (got %d)", who, batch);
    if ((((uintptr_t)x | (uintptr_t)dy | (uintptr_t)u | (uintptr_t)p | (uintptr_t)da | (uintptr_t)db) & 15u) || (((uintptr_t)ids) & 3u))
        return rabit_fail(RABIT_INVALID_ARG, "%s: x, u, dy, p, da and db must be 16-byte aligned, ids 4-byte aligned", who);
    const size_t low = (size_t)batch * A->rank * 4, wa = (size_t)A->count * A->rank * A->n_in, wb = (size_t)A->count * A->rank * A->n_out;
    const Range outs[2] = {{da, wa * 4}, {db, wb * 4}};
    const Range ins[6] = {{x, (size_t)batch * A->n_in * 2}, {dy, (size_t)batch * A->n_out * 2}, {u, low}, {p, low}, {ids, (size_t)batch * 4}, {A->scale, (size_t)A->count * 4}};
    if (outs[0].meets(outs[1])) return rabit_fail(RABIT_INVALID_ARG, "%s: da and db overlap", who);
    for (const Range& o : outs)
        for (const Range& i : ins)
            if (o.meets(i)) return rabit_fail(RABIT_INVALID_ARG, "%s: a gradient overlaps an input", who);
    int dev = -1;
    cudaPointerAttributes attr;
    RABIT_CUDA_TRY(cudaGetDevice(&dev));
    RABIT_CUDA_TRY(cudaPointerGetAttributes(&attr, da));
    if (attr.type != cudaMemoryTypeManaged && (attr.type != cudaMemoryTypeDevice || attr.device != dev))
        return rabit_fail(RABIT_INVALID_ARG, "%s: da is not memory of the current device %d", who, dev);
    if (A->count > 65535) return rabit_fail(RABIT_UNSUPPORTED_SHAPE, "%s: at most 65535 adapters (got %d)", who, A->count);
    cudaStream_t st = (cudaStream_t)stream;
    FactorParams P{};
    P.s[0] = FactorSide{(const __half*)x, p, da, A->n_in, 0};
    P.s[1] = FactorSide{(const __half*)dy, u, db, A->n_out, 0};
    P.ids = ids;
    P.scale = A->scale;
    P.batch = batch;
    P.rank = A->rank;
    P.accumulate = accumulate;
    cudaError_t e = A->rank <= 16 ? launch_factor<1>(P, A->count, st) : A->rank <= 32 ? launch_factor<2>(P, A->count, st)
                  : A->rank <= 64 ? launch_factor<4>(P, A->count, st) : launch_factor<8>(P, A->count, st);
    if (e != cudaSuccess) return rabit_fail(RABIT_CUDA_ERROR, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return RABIT_OK;
}

}  // namespace

extern "C" int rabit_linear_adapted(const rabit_layer* layer, const rabit_adapters* adapters, const void* x, const int* ids, void* y, float* u, int batch, void* stream) {
    rabit_clear_error();
    if (!adapters) return rabit_fail(RABIT_INVALID_ARG, "rabit_linear_adapted: adapters is NULL");
    return adapted_call("rabit_linear_adapted", &layer, &adapters, &x, ids, &y, &u, 1, batch, stream);
}

extern "C" int rabit_linear_group_adapted(const rabit_layer* const* layers, const rabit_adapters* const* adapters, const void* const* xs, const int* ids,
                                          void* const* ys, float* const* us, int n_layers, int batch, void* stream) {
    return adapted_call("rabit_linear_group_adapted", layers, adapters, xs, ids, ys, us, n_layers, batch, stream);
}

extern "C" int rabit_adapter_gradients(const rabit_adapters* adapters, const void* x, const float* u, const void* dy, const float* p, const int* ids,
                                       float* da, float* db, int batch, int accumulate, void* stream) {
    return gradients_call(adapters, x, u, dy, p, ids, da, db, batch, accumulate, stream);
}

extern "C" int rabit_selftest_index_faults(void) {
    rabit_clear_error();
#ifdef RABIT_CHECKED
    unsigned int word = 0, zero = 0;
    RABIT_CUDA_TRY(cudaDeviceSynchronize());
    RABIT_CUDA_TRY(cudaMemcpyFromSymbol(&word, g_index_fault, sizeof word));
    RABIT_CUDA_TRY(cudaMemcpyToSymbol(g_index_fault, &zero, sizeof zero));
    return word ? rabit_fail(RABIT_DEVICE_FAULT, "rabit_selftest_index_faults: an index check of the adapters' kernels failed") : RABIT_OK;
#else
    return rabit_fail(RABIT_UNSUPPORTED_SHAPE, "rabit_selftest_index_faults: this library was built without RABIT_CHECKED");
#endif
}
