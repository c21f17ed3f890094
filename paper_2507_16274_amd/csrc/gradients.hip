// stalloc_clip_gradients: the norm over a list of tensors, and the list scaled to at most that norm.
//
// Bound by device memory: the numbers are read for the norm and read again to be scaled, since no factor is known before
// the last one was read.  The list is host memory and travels as a kernel argument, so there is neither a table to
// upload nor one launch per tensor.  Squares are summed in 64 bits (no square of a finite 32-bit number overflows there, and
// a sum of 10^9 of them is good to 10^-7 times the rounding of the result); every workgroup leaves its sum in a place of its
// own and all of them are added in one order, so the norm does not depend on scheduling.  48 tensors of 25 MiB: 721 us, 5.2 TB/s of two reads and a write (a large copy: 5.1);
// loads or stores past the caches make it slower (737 to 757 us).
#include <math.h>

#include "numbers.h"

namespace stalloc {

constexpr uint32_t kListed = 100;                            // tensors a launch takes: their entries fit the 4 KiB of kernel arguments
constexpr uint32_t kChunk = 8 * 256 * 4;                     // numbers of a tensor that a workgroup takes at a time
constexpr uint32_t kMostBlocks = 2048;                       // workgroups (and partial sums) of a launch

struct Listed {
    const void* data;
    void* out;
    uint64_t count;
    uint32_t chunks_before;                                  // of the tensors before it in the launch
    uint32_t dtype;
};

struct List {
    uint32_t tensors, chunks;
    Listed t[kListed];
};

// The tensor that chunk `c` belongs to: the last one that begins at or before it (entries without numbers begin where the next one does).
__device__ __forceinline__ uint32_t tensor_of(const List& list, uint32_t c)
{
    uint32_t lo = 0, hi = list.tensors - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) / 2;
        if (list.t[mid].chunks_before <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <typename T> __device__ __forceinline__ double chunk_squares(const Listed& t, uint64_t from)
{
    double total = 0.0;
#pragma unroll
    for (uint32_t g = 0; g < kChunk / 2048; ++g) {
        const uint64_t at = from + (g * 256 + threadIdx.x) * 8;
        if (at >= t.count) break;
        const f32x8 v = load_some((const T*)t.data + at, t.count - at > 8 ? 8 : (int)(t.count - at), 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) total = __builtin_fma((double)v[i], (double)v[i], total);
    }
    return total;
}

__global__ void __launch_bounds__(256) list_squares(const List list, double* part)
{
    __shared__ double sums[4];
    double total = 0.0;
    for (uint32_t c = blockIdx.x; c < list.chunks; c += gridDim.x) {
        const Listed& t = list.t[tensor_of(list, c)];
        const uint64_t from = (uint64_t)(c - t.chunks_before) * kChunk;
        if (t.dtype == STALLOC_F32) total += chunk_squares<float>(t, from);
        else if (t.dtype == STALLOC_BF16) total += chunk_squares<bf16>(t, from);
        else total += chunk_squares<f16>(t, from);
    }
    total = wave_sum(total);
    if (lane_id() == 0) sums[wave_id()] = total;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

template <typename T> __device__ __forceinline__ void scale_chunk(const Listed& t, uint64_t from, float factor)
{
#pragma unroll
    for (uint32_t g = 0; g < kChunk / 2048; ++g) {
        const uint64_t at = from + (g * 256 + threadIdx.x) * 8;
        if (at >= t.count) break;
        const int n = t.count - at > 8 ? 8 : (int)(t.count - at);
        store_some((T*)t.out + at, n, load_some((const T*)t.data + at, n, 0.f) * factor);
    }
}

// Every workgroup adds all partial sums up by itself (in the same order, so all get the same factor): cheaper than a launch between.
__global__ void __launch_bounds__(256) list_scale(const List list, const double* __restrict__ part, uint32_t parts, float max_norm, float* norm, float* factor)
{
    __shared__ double sums[4];
    double total = 0.0;
    for (uint32_t i = threadIdx.x; i < parts; i += 256) total += part[i];
    total = wave_sum(total);
    if (lane_id() == 0) sums[wave_id()] = total;
    __syncthreads();
    const double root = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3]));
    float f = 1.f;
    if (root > (double)max_norm && (float)root < INFINITY) f = (float)((double)max_norm / root);
    if (blockIdx.x == 0 && threadIdx.x == 0) { *norm = (float)root; *factor = f; }
    for (uint32_t i = blockIdx.x; i < list.chunks; i += gridDim.x) {
        const uint32_t c = list.chunks - 1 - i;              // last chunks first: they are what the first kernel left in the caches
        const Listed& t = list.t[tensor_of(list, c)];
        const uint64_t from = (uint64_t)(c - t.chunks_before) * kChunk;
        if (!t.out || (f == 1.f && t.out == t.data)) continue;
        if (t.dtype == STALLOC_F32) scale_chunk<float>(t, from, f);
        else if (t.dtype == STALLOC_BF16) scale_chunk<bf16>(t, from, f);
        else scale_chunk<f16>(t, from, f);
    }
}

}  // namespace stalloc

using namespace stalloc;

namespace {

// Entries first .. of the caller's list as the argument of one launch; returns how many were taken.
uint32_t fill(List* list, const stalloc_tensor* tensors, uint32_t k, uint32_t first)
{
    list->tensors = 0;
    uint64_t chunks = 0;
    uint32_t i = first;
    for (; i < k && list->tensors < kListed; ++i) {
        const uint64_t more = (tensors[i].count + kChunk - 1) / kChunk;
        if (chunks + more > 0x40000000u && list->tensors) break;
        list->t[list->tensors++] = {tensors[i].data, tensors[i].out, tensors[i].count, (uint32_t)chunks, (uint32_t)tensors[i].dtype};
        chunks += more;
    }
    list->chunks = (uint32_t)chunks;
    return i - first;
}

uint32_t blocks_of(const List& list) { return list.chunks < kMostBlocks ? (list.chunks ? list.chunks : 1) : kMostBlocks; }

}  // namespace

extern "C" int stalloc_clip_gradients(const stalloc_tensor* tensors, uint32_t k, float max_norm, float* norm, float* factor,
                                      void* workspace, size_t* workspace_bytes, void* hip_stream)
{
    if (!tensors || k == 0 || !(max_norm >= 0.f) || !workspace_bytes) return STALLOC_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < k; ++i) {
        const stalloc_tensor& t = tensors[i];
        if (t.dtype > STALLOC_F16 || t.count >= (1ull << 42)) return STALLOC_ERR_INVALID_ARG;
        const size_t size = bytes_of((uint32_t)t.dtype);
        if ((t.count && !t.data) || !aligned(t.data, size) || !aligned(t.out, size)) return STALLOC_ERR_INVALID_ARG;
    }
    List list;
    size_t parts = 0;
    for (uint32_t at = 0; at < k;) {
        at += fill(&list, tensors, k, at);
        parts += blocks_of(list);
    }
    Carver cv(workspace);
    double* part = cv.take<double>(parts);
    if (!workspace) { *workspace_bytes = cv.used; return STALLOC_OK; }
    if (!norm || !factor || *workspace_bytes < cv.used || !aligned(workspace, kAlign)) return STALLOC_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    begin_launches();
    size_t done = 0;
    for (uint32_t at = 0; at < k;) {
        at += fill(&list, tensors, k, at);
        hipLaunchKernelGGL(list_squares, dim3(blocks_of(list)), dim3(256), 0, stream, list, part + done);
        done += blocks_of(list);
    }
    for (uint32_t at = 0; at < k;) {
        at += fill(&list, tensors, k, at);
        hipLaunchKernelGGL(list_scale, dim3(blocks_of(list)), dim3(256), 0, stream, list, part, (uint32_t)parts, max_norm, norm, factor);
    }
    return launched();
}
