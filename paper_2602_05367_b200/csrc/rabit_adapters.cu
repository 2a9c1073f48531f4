// Low-rank adapters of many requests beside a layer, and the gradients of their factors.
//
//   u[t] = A[id_t] x[t],   y[t] = layer(x[t]) + scale[id_t] * B[id_t]^T u[t]
//   da[i] = scale[i] * sum_{t: id_t = i} p[t] x[t]^T,   db[i] = scale[i] * sum_{t: id_t = i} u[t] dy[t]^T
//
// Every factor is `rank` rows along a side of the layer, so both products of the forward pass and of the input gradient are the same two kernels.
#include <cuda_fp16.h>

#include <algorithm>
#include <cstring>

#include "rabit_internal.h"

namespace {

constexpr int kThreads = 256;

// u[t][j] = sum_n A[id][j][n] x[t][n]: one CTA per row, a warp per rank row.
__global__ void __launch_bounds__(kThreads) narrow_kernel(const __half* __restrict__ x, const int* __restrict__ ids, const __half* __restrict__ a, float* __restrict__ u, int count, int rank, int n) {
    const int t = blockIdx.x, id = ids[t], lane = threadIdx.x & 31;
    const bool some = id >= 0 && id < count;
    const uint4* xr = reinterpret_cast<const uint4*>(x + (size_t)t * n);
    for (int j = threadIdx.x >> 5; j < rank; j += kThreads / 32) {
        float sum = 0.f;
        if (some) {
            const uint4* ar = reinterpret_cast<const uint4*>(a + ((size_t)id * rank + j) * n);
            for (int i = lane; i < n / 8; i += 32) {
                const uint4 av = ar[i], xv = xr[i];
                const __half2 *ah = reinterpret_cast<const __half2*>(&av), *xh = reinterpret_cast<const __half2*>(&xv);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float2 af = __half22float2(ah[q]), xf = __half22float2(xh[q]);
                    sum = fmaf(af.x, xf.x, sum);
                    sum = fmaf(af.y, xf.y, sum);
                }
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (lane == 0) u[(size_t)t * rank + j] = sum;
    }
}

// y[t][m] += scale[id] * sum_j B[id][j][m] u[t][j]: a thread per output.
__global__ void __launch_bounds__(kThreads) widen_kernel(const float* __restrict__ u, const int* __restrict__ ids, const __half* __restrict__ b, const float* __restrict__ scale, __half* __restrict__ y, int count, int rank, int m_all) {
    const int t = blockIdx.y, id = ids[t], m = blockIdx.x * kThreads + threadIdx.x;
    if (id < 0 || id >= count || m >= m_all) return;
    float sum = 0.f;
    for (int j = 0; j < rank; ++j) sum = fmaf(__half2float(b[((size_t)id * rank + j) * m_all + m]), u[(size_t)t * rank + j], sum);
    __half* at = y + (size_t)t * m_all + m;
    *at = __float2half_rn(fmaf(scale[id], sum, __half2float(*at)));
}

// out[i][j][d] (+)= scale[i] * sum over the adapter's rows of low[t][j] v[t][d]: a thread per element.
__global__ void __launch_bounds__(kThreads) factor_kernel(const __half* __restrict__ v, const float* __restrict__ low, const int* __restrict__ ids, const float* __restrict__ scale, float* __restrict__ out, int batch, int rank, int side, int accumulate) {
    const int d = blockIdx.x * kThreads + threadIdx.x, j = blockIdx.y, i = blockIdx.z;
    if (d >= side) return;
    float total = 0.f;
    for (int t0 = 0; t0 < batch; t0 += 64) {                     // (partial sums of 64 rows: the rounding error of a long sum stays small)
        float sum = 0.f;
        for (int t = t0; t < min(batch, t0 + 64); ++t)
            if (ids[t] == i) sum = fmaf(low[(size_t)t * rank + j], __half2float(v[(size_t)t * side + d]), sum);
        total += sum;
    }
    float* at = out + ((size_t)i * rank + j) * side + d;
    *at = (accumulate ? *at : 0.f) + scale[i] * total;
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

int adapted_call(const char* who, const rabit_layer* const* layers, const rabit_adapters* const* adapters, const void* const* xs, const int* ids,
                 void* const* ys, float* const* us, int n_layers, int batch, void* stream) {
    rabit_clear_error();
    if (!layers || !adapters || !xs || !ys || !us) return rabit_fail(RABIT_INVALID_ARG, "%s: null array", who);
    if (n_layers < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: n_layers must be >= 1 (got %d)", who, n_layers);
    if (batch < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: batch must be >= 1 (got %d)", who, batch);
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
    int rc = n_layers == 1 ? rabit_linear(layers[0], xs[0], ys[0], batch, stream) : rabit_linear_group(layers, xs, ys, n_layers, batch, stream);
    if (rc != RABIT_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    for (int l = 0; l < n_layers; ++l) {
        const rabit_adapters* A = adapters[l];
        if (!A) continue;
        narrow_kernel<<<batch, kThreads, 0, st>>>((const __half*)xs[l], ids, (const __half*)A->a, us[l], A->count, A->rank, A->n_in);
        for (int t0 = 0; t0 < batch; t0 += 32768)
            widen_kernel<<<dim3((A->n_out + kThreads - 1) / kThreads, std::min(batch - t0, 32768)), kThreads, 0, st>>>(us[l] + (size_t)t0 * A->rank, ids + t0, (const __half*)A->b, A->scale,
                                                                                                            (__half*)ys[l] + (size_t)t0 * A->n_out, A->count, A->rank, A->n_out);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return rabit_fail(RABIT_CUDA_ERROR, "%s: launch failed: %s", who, cudaGetErrorString(e));
    }
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
    if (A->count > 65535) return rabit_fail(RABIT_UNSUPPORTED_SHAPE, "%s: at most 65535 adapters (got %d)", who, A->count);
    cudaStream_t st = (cudaStream_t)stream;
    factor_kernel<<<dim3((A->n_in + kThreads - 1) / kThreads, A->rank, A->count), kThreads, 0, st>>>((const __half*)x, p, ids, A->scale, da, batch, A->rank, A->n_in, accumulate);
    factor_kernel<<<dim3((A->n_out + kThreads - 1) / kThreads, A->rank, A->count), kThreads, 0, st>>>((const __half*)dy, u, ids, A->scale, db, batch, A->rank, A->n_out, accumulate);
    cudaError_t e = cudaGetLastError();
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
