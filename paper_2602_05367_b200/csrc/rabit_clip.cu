// The global norm over many gradient tensors, and clipping by it.
//
//   norm = sqrt(sum g^2),   g * min(1, max_norm / (norm + 1e-6))
//
// Two kernels: partial sums of squares, one per CTA; then every CTA adds all of them in the same order, which is cheaper than a third
// launch, and scales its share.  Bound: memory.  40 M elements in 448 tensors, out of place: 74 us, 29 for the first reading (5.5 TB/s) and 45 for the second with
// the writing (7.1); 49 would do with the second reading free, but little of 160 MB is still in L2 by then (streaming stores and the reversed order change
// nothing).  0.65 M elements: 4.8 us, two launches' latency.
// Squares are taken and summed in 64 bits: an fp32 gradient of 1e20 has no fp32 square, and the conversion and the double add cost less than the bytes.
#include <algorithm>
#include <memory>
#include <new>
#include <utility>
#include <vector>

#include "rabit_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr size_t kChunk = 4096;                       // elements that a CTA takes at a time
constexpr int kMaxGrid = 2048;

struct Chunk {                                        // a piece of one tensor
    const float* src;
    float* dst;
    uint32_t n, aligned;                              // aligned: both pointers on 16 bytes
};
constexpr int kFours = (int)(kChunk / 4 / kThreads);  // 16-byte accesses of a thread to a chunk
static_assert((size_t)kFours * 4 * kThreads == kChunk, "a chunk is whole accesses of all threads");

// a thread's share of a chunk, 4 * kFours elements, zero behind its end; `store` puts them back
__device__ __forceinline__ void load_chunk(const Chunk& c, float (&v)[4 * kFours]) {
#pragma unroll
    for (int i = 0; i < kFours; ++i) {
        const uint32_t at = 4u * (i * kThreads + threadIdx.x);
        if (c.aligned && at + 4 <= c.n) {
            const float4 w = *reinterpret_cast<const float4*>(c.src + at);
            v[4 * i] = w.x; v[4 * i + 1] = w.y; v[4 * i + 2] = w.z; v[4 * i + 3] = w.w;
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) v[4 * i + q] = at + q < c.n ? c.src[at + q] : 0.f;
        }
    }
}
__device__ __forceinline__ void store_chunk(const Chunk& c, const float (&v)[4 * kFours]) {
#pragma unroll
    for (int i = 0; i < kFours; ++i) {
        const uint32_t at = 4u * (i * kThreads + threadIdx.x);
        if (c.aligned && at + 4 <= c.n) {
            *reinterpret_cast<float4*>(c.dst + at) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (at + q < c.n) c.dst[at + q] = v[4 * i + q];
        }
    }
}

__device__ __forceinline__ double block_sum(double v, double* warps) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += warps[w];
    return s;
}

__global__ void __launch_bounds__(kThreads) squares_kernel(const Chunk* __restrict__ chunks, int n_chunks, double* __restrict__ partial) {
    __shared__ double warps[kThreads / 32];
    double sum = 0.0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    Chunk next = (int)blockIdx.x < n_chunks ? chunks[blockIdx.x] : Chunk{};
    for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const Chunk ch = next;
        if (c + (int)gridDim.x < n_chunks) next = chunks[c + gridDim.x];
        float v[4 * kFours];
        load_chunk(ch, v);
#pragma unroll
        for (int i = 0; i < 4 * kFours; ++i) sum = fma((double)v[i], (double)v[i], sum);
    }
    sum = block_sum(sum, warps);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kThreads) scale_kernel(const Chunk* __restrict__ chunks, int n_chunks, const double* partial, double max_norm, float* norm_out) {
    __shared__ double warps[kThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum = 0.0;
    // (from L2, and not as data that stays the same while this kernel runs: it starts while the sums are being written)
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) sum += __ldcg(partial + i);
    const double norm = sqrt(block_sum(sum, warps));
    double f = max_norm / (norm + 1e-6);
    if (f > 1.0) f = 1.0;                             // (a NaN stays)
    const float factor = (float)f;
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    // from the last chunk to the first: what was read last is still in L2
    Chunk next = (int)blockIdx.x < n_chunks ? chunks[n_chunks - 1 - blockIdx.x] : Chunk{};
    for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const Chunk ch = next;
        if (c + (int)gridDim.x < n_chunks) next = chunks[n_chunks - 1 - c - gridDim.x];
        if (ch.dst == ch.src && factor == 1.f) continue;
        float v[4 * kFours];
        load_chunk(ch, v);
#pragma unroll
        for (int i = 0; i < 4 * kFours; ++i) v[i] *= factor;
        store_chunk(ch, v);
    }
}

size_t chunks_of(const size_t* counts, int n) {
    size_t total = 0;
    for (int i = 0; i < n; ++i) total += (counts[i] + kChunk - 1) / kChunk;
    return total;
}

}  // namespace

struct Span {
    uintptr_t at, end;
    bool written;
};

struct rabit_gradients {
    int device, n_chunks, grid;
    const Chunk* chunks;
    double* partial;
    std::vector<Span> spans;                          // all memory of a call, by its start
};

// table of chunks | one partial sum per CTA
extern "C" size_t rabit_gradients_bytes(const size_t* counts, int n) {
    if (!counts || n < 1) return 0;
    return rabit_align256(chunks_of(counts, n) * sizeof(Chunk)) + kMaxGrid * sizeof(double);
}

static int bind_call(const float* const* tensors, float* const* outs, const size_t* counts, int n, void* dev_buf, size_t dev_bytes, void* stream, rabit_gradients** out) {
    const char* who = "rabit_gradients_bind";
    rabit_clear_error();
    if (!out) return rabit_fail(RABIT_INVALID_ARG, "%s: out is NULL", who);
    *out = nullptr;
    if (!tensors || !counts || !dev_buf) return rabit_fail(RABIT_INVALID_ARG, "%s: null pointer", who);
    if (n < 1) return rabit_fail(RABIT_INVALID_ARG, "%s: n must be >= 1 (got %d)", who, n);
    if (((uintptr_t)dev_buf & 255u) != 0) return rabit_fail(RABIT_INVALID_ARG, "%s: dev_buf must be 256-byte aligned", who);
    for (int i = 0; i < n; ++i) {
        if (counts[i] > ((size_t)1 << 40)) return rabit_fail(RABIT_INVALID_ARG, "%s: tensor %d has %zu elements", who, i, counts[i]);
        if (counts[i] && (!tensors[i] || (outs && !outs[i]))) return rabit_fail(RABIT_INVALID_ARG, "%s: null tensor %d", who, i);
        if (counts[i] && ((((uintptr_t)tensors[i]) & 3u) || (outs && (((uintptr_t)outs[i]) & 3u)))) return rabit_fail(RABIT_INVALID_ARG, "%s: tensor %d is misaligned", who, i);
    }
    const size_t n_chunks = chunks_of(counts, n);
    if (n_chunks > 0x7FFFFFFFu) return rabit_fail(RABIT_UNSUPPORTED_SHAPE, "%s: too many elements", who);
    const size_t need = rabit_gradients_bytes(counts, n), table_bytes = rabit_align256(n_chunks * sizeof(Chunk));
    if (dev_bytes < need) return rabit_fail(RABIT_BUFFER_TOO_SMALL, "%s: dev_buf holds %zu bytes, need %zu", who, dev_bytes, need);
    // what is written overlaps nothing else: a sweep over all ranges by their starts
    std::vector<Span> spans;
    spans.push_back({(uintptr_t)dev_buf, (uintptr_t)dev_buf + need, true});
    for (int i = 0; i < n; ++i) {
        if (!counts[i]) continue;
        const uintptr_t s = (uintptr_t)tensors[i], d = outs ? (uintptr_t)outs[i] : s;
        if (s != d) spans.push_back({s, s + counts[i] * 4, false});
        spans.push_back({d, d + counts[i] * 4, true});
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
    uintptr_t end_all = 0, end_written = 0;
    for (const Span& s : spans) {
        if ((s.written && end_all > s.at) || end_written > s.at) return rabit_fail(RABIT_INVALID_ARG, "%s: an output overlaps another tensor or dev_buf", who);
        end_all = std::max(end_all, s.end);
        if (s.written) end_written = std::max(end_written, s.end);
    }
    cudaPointerAttributes attr;
    RABIT_CUDA_TRY(cudaPointerGetAttributes(&attr, dev_buf));
    if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged) return rabit_fail(RABIT_INVALID_ARG, "%s: dev_buf is not device memory", who);
    // (a captured copy would read the table again at every replay, when it is gone)
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    RABIT_CUDA_TRY(cudaStreamIsCapturing((cudaStream_t)stream, &capturing));
    if (capturing != cudaStreamCaptureStatusNone) return rabit_fail(RABIT_INVALID_ARG, "%s: the stream is being captured", who);
    std::vector<Chunk> table;
    table.reserve(n_chunks);
    for (int i = 0; i < n; ++i)
        for (size_t at = 0; at < counts[i]; at += kChunk) {
            const float* src = tensors[i] + at;
            float* dst = outs ? outs[i] + at : const_cast<float*>(src);
            table.push_back(Chunk{src, dst, (uint32_t)std::min(kChunk, counts[i] - at), (uint32_t)(((uintptr_t)src | (uintptr_t)dst) % 16 == 0)});
        }
    // The table is in place when this returns, so a call may come on any stream: one that read it too early would take whatever is there for addresses.
    if (!table.empty()) RABIT_CUDA_TRY(cudaMemcpyAsync(dev_buf, table.data(), table.size() * sizeof(Chunk), cudaMemcpyHostToDevice, (cudaStream_t)stream));
    RABIT_CUDA_TRY(cudaStreamSynchronize((cudaStream_t)stream));
    int sms = 0;
    RABIT_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, attr.device));
    std::unique_ptr<rabit_gradients> R(new rabit_gradients);
    R->device = attr.device;
    R->n_chunks = (int)n_chunks;
    R->grid = (int)std::max<size_t>(1, std::min<size_t>(n_chunks, std::min(8 * sms, kMaxGrid)));
    R->chunks = (const Chunk*)dev_buf;
    R->partial = (double*)((char*)dev_buf + table_bytes);
    R->spans = std::move(spans);
    *out = R.release();
    return RABIT_OK;
}

extern "C" int rabit_gradients_bind(const float* const* tensors, float* const* outs, const size_t* counts, int n, void* dev_buf, size_t dev_bytes, void* stream, rabit_gradients** out) {
    return rabit_guarded("rabit_gradients_bind", [&] { return bind_call(tensors, outs, counts, n, dev_buf, dev_bytes, stream, out); });
}

extern "C" int rabit_clip_gradients(const rabit_gradients* R, float max_norm, float* norm_out, void* stream) {
    const char* who = "rabit_clip_gradients";
    rabit_clear_error();
    if (!R || !norm_out || (((uintptr_t)norm_out) & 3u)) return rabit_fail(RABIT_INVALID_ARG, "%s: gradients or norm_out is NULL or misaligned", who);
    if (!(max_norm > 0.f) || !(max_norm <= 3.402823466e38f)) return rabit_fail(RABIT_INVALID_ARG, "%s: max_norm must be positive and finite", who);
    for (const Span& s : R->spans)
        if (rabit_ranges_overlap((const void*)s.at, s.end - s.at, norm_out, 4)) return rabit_fail(RABIT_INVALID_ARG, "%s: norm_out lies in a gradient, an output or dev_buf", who);
    int dev = -1;
    RABIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev != R->device) return rabit_fail(RABIT_INVALID_ARG, "%s: the gradients live on device %d but device %d is current", who, R->device, dev);
    cudaStream_t st = (cudaStream_t)stream;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)R->grid);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, squares_kernel, R->chunks, R->n_chunks, R->partial);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, scale_kernel, R->chunks, R->n_chunks, (const double*)R->partial, (double)max_norm, norm_out);
    if (e != cudaSuccess) return rabit_fail(RABIT_CUDA_ERROR, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return RABIT_OK;
}

extern "C" int rabit_gradients_free(rabit_gradients* R) {
    rabit_clear_error();
    delete R;
    return RABIT_OK;
}
