// stalloc_token_logprobs, stalloc_token_logprobs_backward: the softmax over a vocabulary without its probabilities.
//
//     m = max x,  Z = sum exp(x - m),  A = sum exp(x - m) (x - m):   lse = m + ln Z,  log p_y = x_y - lse,  H = ln Z - A / Z
//     dx_j = g ([j = y] - p_j) - h p_j (ln p_j + H)
//
// One pass over the logits with a running maximum: eight numbers at a time raise m, and Z and A are brought to the new m by
// one factor.  Sums are kept in units of log 2, (x - m) log2(e), for the hardware's exponential.  Few rows are cut
// into parts so that the whole chip reads, and a wave per row joins them.
//
// The most likely tokens cost no second pass: a thread remembers which group of eight gave it its maximum (the running maximum
// it needs anyway).  The largest of the workgroup's 256 maxima is the row's first; the thread that owned it then offers its next best,
// for which its numbers alone (a 256th of the row) are looked at again.
#include <math.h>

#include "numbers.h"

namespace stalloc {

constexpr uint32_t kMostTop = 64;
constexpr uint32_t kMostParts = 64;
constexpr int kLpThreads = 256;

// A number and its place as one integer: larger numbers first, then lower places; 0 is below all.  -0 counts as 0.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t place)
{
    const uint32_t b = as_bits(x + 0.f);
    const uint32_t order = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return ((uint64_t)order << 32) | (uint32_t)~place;
}
__device__ __forceinline__ uint32_t place_of(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ float number_of(uint64_t key)
{
    const uint32_t order = (uint32_t)(key >> 32);
    return as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

// Maximum, sum of 2^t and of t 2^t over some numbers, t = (x - m) log2(e); nothing yet: m the lowest finite number.
struct Softmax {
    float m, z, a;
};
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ Softmax of_nothing() { return {kLowest, 0.f, 0.f}; }

// 2^t and what multiplies it in A: -infinity times 0 must not arise, a NaN must not vanish (it is in 2^t).
__device__ __forceinline__ float lowest_t(float t) { return fmaxf(t, -1e4f); }

__device__ __forceinline__ void rebase(Softmax& s, float m)
{
    const float t = lowest_t((s.m - m) * kLog2e), f = exp2_fast(t);
    s.a = (s.a + s.z * t) * f;
    s.z *= f;
    s.m = m;
}

__device__ __forceinline__ void join(Softmax& s, Softmax o)
{
    const float m = fmaxf(s.m, o.m);
    rebase(s, m);
    rebase(o, m);
    s.z += o.z;
    s.a += o.a;
}

__device__ __forceinline__ Softmax from_lane_xor(const Softmax& s, int step)
{
    Softmax o;
    o.m = __shfl_xor(s.m, step, kWave);
    o.z = __shfl_xor(s.z, step, kWave);
    o.a = __shfl_xor(s.a, step, kWave);
    return o;
}

__device__ __forceinline__ Softmax with_eight(Softmax s, f32x8 v)
{
    const float m = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    rebase(s, fmaxf(s.m, m));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = (v[i] - s.m) * kLog2e, e = exp2_fast(d);
        s.z += e;
        s.a = __builtin_fmaf(e, lowest_t(d), s.a);
    }
    return s;
}

// Over the workgroup's threads, in all of them and in one order.
__device__ __forceinline__ Softmax join_workgroup(Softmax s, Softmax* waves)
{
#pragma unroll
    for (int step = 1; step < kWave; step <<= 1) join(s, from_lane_xor(s, step));
    if (lane_id() == 0) waves[wave_id()] = s;
    __syncthreads();
    s = waves[0];
#pragma unroll
    for (int w = 1; w < kLpThreads / kWave; ++w) join(s, waves[w]);
    return s;
}

struct LogprobArgs {
    uint32_t rows, vocabulary, top, parts, part_width;       // part_width: columns of a part, a multiple of 8
    const void* logits;
    uint64_t row_stride;
    const int32_t* tokens;
    float* logprob;
    float* entropy;
    float* lse;
    int32_t* top_tokens;
    float* top_logprobs;
    uint32_t* status;
    Softmax* part;                                           // [rows][parts]
    uint64_t* keys;                                          // [rows][parts][top]
};

template <typename T> __device__ __forceinline__ void finish_row(const LogprobArgs& a, uint32_t row, const Softmax& s)
{
    const float ln_z = logf(s.z);                            // (log 0 = -infinity: nothing can occur)
    const int32_t token = a.tokens[row];
    float lp = 0.f;
    if (token >= 0 && token < (int32_t)a.vocabulary) lp = s.z == 0.f ? -INFINITY : ((float)((const T*)a.logits)[row * a.row_stride + token] - s.m) - ln_z;
    a.logprob[row] = lp;
    a.entropy[row] = s.z == 0.f ? 0.f : ln_z - s.a / s.z * kLn2;
    a.lse[row] = s.z == 0.f ? -INFINITY : s.m + ln_z;
}

__device__ __forceinline__ void put_top(const LogprobArgs& a, uint32_t row, uint32_t rank, uint64_t key, const Softmax& s)
{
    const uint64_t at = (uint64_t)row * a.top + rank;
    a.top_tokens[at] = (int32_t)place_of(key);
    a.top_logprobs[at] = s.z == 0.f ? -INFINITY : (number_of(key) - s.m) - logf(s.z);
}

// The first workgroup looks at all tokens and writes the status: neither a launch to clear it nor atomics.
__device__ __forceinline__ void check_tokens(const int32_t* __restrict__ tokens, uint32_t rows, uint32_t vocabulary, uint32_t* status, uint32_t* words)
{
    uint32_t bad = 0;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < rows; i += kLpThreads) bad |= tokens[i] >= (int32_t)vocabulary;
    const uint64_t any = __ballot(bad != 0);
    if (lane_id() == 0) words[wave_id()] = any != 0;
    __syncthreads();
    if (threadIdx.x == 0) *status = words[0] | words[1] | words[2] | words[3] ? STALLOC_ERR_BAD_TOKEN : STALLOC_OK;
}

// A workgroup takes one part of one row.
template <typename T> __global__ void __launch_bounds__(kLpThreads) lp_row(LogprobArgs a)
{
    __shared__ Softmax waves[kLpThreads / kWave];
    __shared__ uint64_t best[kLpThreads];
    __shared__ uint32_t words[kLpThreads / kWave];
    if (blockIdx.x == 0) check_tokens(a.tokens, a.rows, a.vocabulary, a.status, words);
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts, t = threadIdx.x;
    const T* x = (const T*)a.logits + row * a.row_stride;
    const uint32_t from = part * a.part_width, to = umin(a.vocabulary, from + a.part_width);   // (the last parts may be empty: from >= to)
    Softmax s = of_nothing();
    float most = -INFINITY;                                  // this thread's maximum, and where it was met first
    uint32_t group = from + t * 8;
    for (uint32_t at = from + t * 8; at < to; at += kLpThreads * 8) {
        const f32x8 v = load_some(x + at, (int)(to - at), -INFINITY);
        const float m = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
        if (m > most) group = at;
        most = fmaxf(most, m);
        s = with_eight(s, v);
    }
    if (a.top) {
        uint64_t k = 0;
        if (group < to) {
            const f32x8 v = load_some(x + group, (int)(to - group), -INFINITY);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (group + i < to) k = umax64(k, key_of(v[i], group + i));
        }
        best[t] = k;
    }
    s = join_workgroup(s, waves);
    if (wave_id() != 0) return;
    if (a.parts > 1) {
        if (t == 0) a.part[blockIdx.x] = s;
    } else if (t == 0) {
        finish_row<T>(a, row, s);
    }
    uint64_t mine[kLpThreads / kWave];                       // lane l looks after the threads 4 l .. 4 l + 3
#pragma unroll
    for (int i = 0; i < kLpThreads / kWave; ++i) mine[i] = a.top ? best[t * (kLpThreads / kWave) + i] : 0;
    for (uint32_t rank = 0; rank < a.top; ++rank) {
        uint64_t k = mine[0];
#pragma unroll
        for (int i = 1; i < kLpThreads / kWave; ++i) k = umax64(k, mine[i]);
        k = wave_max64(k);
        if (a.parts > 1) { if (t == 0) a.keys[(uint64_t)blockIdx.x * a.top + rank] = k; }
        else if (t == 0) put_top(a, row, rank, k, s);
        if (rank + 1 == a.top) break;
        const uint32_t owner = ((place_of(k) - from) / 8) % kLpThreads;
        uint64_t next = 0;                                   // the owner's largest key below the one taken
        for (uint32_t at = from + (owner + t * kLpThreads) * 8; at < to; at += kWave * kLpThreads * 8) {
            const f32x8 v = load_some(x + at, (int)(to - at), -INFINITY);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t other = key_of(v[i], at + i);
                if (at + i < to && other < k) next = umax64(next, other);
            }
        }
        next = wave_max64(next);
        if (t == owner / (kLpThreads / kWave)) {
#pragma unroll
            for (int i = 0; i < kLpThreads / kWave; ++i)
                if (owner % (kLpThreads / kWave) == (uint32_t)i) mine[i] = next;
        }
    }
}

// A wave joins the parts of a row (at most 64, a lane each) and picks the row's most likely tokens from theirs, which every part lists
// in descending order: a lane holds the first one not taken yet.
template <typename T> __global__ void __launch_bounds__(kWave) lp_join(LogprobArgs a)
{
    const uint32_t row = blockIdx.x, lane = lane_id();
    Softmax s = of_nothing();
    if (lane < a.parts) s = a.part[(uint64_t)row * a.parts + lane];
#pragma unroll
    for (int step = 1; step < kWave; step <<= 1) join(s, from_lane_xor(s, step));
    if (lane == 0) finish_row<T>(a, row, s);
    const uint64_t* list = a.keys + ((uint64_t)row * a.parts + lane) * a.top;
    uint32_t taken = 0;
    uint64_t k = lane < a.parts && a.top ? list[0] : 0;
    for (uint32_t rank = 0; rank < a.top; ++rank) {
        const uint64_t first = wave_max64(k);
        if (lane == 0) put_top(a, row, rank, first, s);
        if (lane < a.parts && k == first) k = ++taken < a.top ? list[taken] : 0;
    }
}

struct LogprobBackwardArgs {
    uint32_t rows, vocabulary, chunks;
    const void* logits;
    uint64_t row_stride;
    const int32_t* tokens;
    const float* lse;
    const float* entropy;
    const float* d_logprob;
    const float* d_entropy;
    void* d_logits;
    uint64_t d_row_stride;
    uint32_t* status;
};

constexpr uint32_t kLpChunk = kLpThreads * 8 * 4;

constexpr float kFarLse = 256.f;

// A workgroup takes a chunk of a row.  Each number is read before the thread that read it writes its gradient, which may go to the same place.
// An lse beyond 256 (logits around a type's lowest value, say) says too little in 32 bits: the first workgroup of such a row then
// sums it up again and writes all of it.
template <typename T> __global__ void __launch_bounds__(kLpThreads) lp_backward(LogprobBackwardArgs a)
{
    __shared__ uint32_t words[kLpThreads / kWave];
    __shared__ Softmax waves[kLpThreads / kWave];
    if (blockIdx.x == 0) check_tokens(a.tokens, a.rows, a.vocabulary, a.status, words);
    const uint32_t row = blockIdx.x / a.chunks;
    uint32_t chunk = blockIdx.x % a.chunks, end = chunk + 1;
    const T* x = (const T*)a.logits + row * a.row_stride;
    T* d = (T*)a.d_logits + row * a.d_row_stride;
    const int32_t token = a.tokens[row];
    const float lse = a.lse[row], h = a.d_entropy ? a.d_entropy[row] : 0.f, entropy = h != 0.f ? a.entropy[row] : 0.f;
    const float g = token >= 0 ? a.d_logprob[row] : 0.f;
    const bool nothing = lse == -INFINITY;                   // a row in which nothing can occur: no gradient
    float m = lse, ln_z = 0.f;
    if (fabsf(lse) > kFarLse && fabsf(lse) < INFINITY) {
        if (chunk != 0) return;
        end = a.chunks;
        Softmax s = of_nothing();
        for (uint32_t at = threadIdx.x * 8; at < a.vocabulary; at += kLpThreads * 8) s = with_eight(s, load_some(x + at, (int)(a.vocabulary - at), -INFINITY));
        s = join_workgroup(s, waves);
        m = s.m;
        ln_z = logf(s.z);
    }
    for (; chunk < end; ++chunk)
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t at = chunk * kLpChunk + (u * kLpThreads + threadIdx.x) * 8;
            if (at >= a.vocabulary) break;
            const int n = (int)(a.vocabulary - at);
            const f32x8 v = load_some(x + at, n, -INFINITY);
            f32x8 out;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float l = (v[i] - m) - ln_z, p = exp2_fast(l * kLog2e);
                float w = g;
                if (h != 0.f) w += h * (fmaxf(l, -1e4f) + entropy);
                float r = -p * w;
                if (at + i == (uint32_t)token) r += g;
                out[i] = nothing ? 0.f : r;
            }
            store_some(d + at, n, out);
        }
}

// Parts of a row: as many as give the chip eight workgroups per CU, of at least 4096 numbers each.
struct LpShape {
    uint32_t parts, part_width;
};
inline LpShape lp_shape(uint32_t rows, uint32_t vocabulary)
{
    const uint32_t wanted = (2048 + rows - 1) / rows, most = (vocabulary + 4095) / 4096;
    uint32_t parts = umin_host(umin_host(wanted, most), kMostParts);
    const uint32_t width = (uint32_t)((((uint64_t)vocabulary + parts - 1) / parts + 7) / 8 * 8);
    return {parts, width};
}

}  // namespace stalloc

using namespace stalloc;

namespace {

bool lp_sizes_ok(uint32_t dtype, uint32_t rows, uint32_t vocabulary)
{
    return dtype <= STALLOC_F16 && rows >= 1 && rows < 0x1000000u && vocabulary >= 1 && vocabulary < 0x40000000u;
}

}  // namespace

extern "C" int stalloc_token_logprobs(uint32_t dtype, uint32_t rows, uint32_t vocabulary, const void* logits, uint64_t row_stride,
                                      const int32_t* tokens, uint32_t top, float* logprob, float* entropy, float* lse,
                                      int32_t* top_tokens, float* top_logprobs, uint32_t* device_status, void* workspace,
                                      size_t* workspace_bytes, void* hip_stream)
{
    if (!lp_sizes_ok(dtype, rows, vocabulary) || top > kMostTop || top > vocabulary || !workspace_bytes) return STALLOC_ERR_INVALID_ARG;
    const LpShape shape = lp_shape(rows, vocabulary);
    Carver cv(workspace);
    Softmax* part = cv.take<Softmax>(shape.parts > 1 ? (size_t)rows * shape.parts : 1);
    uint64_t* keys = cv.take<uint64_t>(shape.parts > 1 ? (size_t)rows * shape.parts * top : 0);
    if (!workspace) { *workspace_bytes = cv.used; return STALLOC_OK; }
    if (!logits || !tokens || !logprob || !entropy || !lse || !device_status || (top && (!top_tokens || !top_logprobs)) ||
        *workspace_bytes < cv.used || !aligned(workspace, kAlign) || !aligned(logits, bytes_of(dtype)))
        return STALLOC_ERR_INVALID_ARG;
    const LogprobArgs a = {rows, vocabulary, top, shape.parts, shape.part_width, logits, row_stride, tokens, logprob, entropy, lse,
                           top_tokens, top_logprobs, device_status, part, keys};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(lp_row<T>, dim3(rows * shape.parts), dim3(kLpThreads), 0, stream, a);
        if (shape.parts > 1) hipLaunchKernelGGL(lp_join<T>, dim3(rows), dim3(kWave), 0, stream, a);
    });
    return launched();
}

extern "C" int stalloc_token_logprobs_backward(uint32_t dtype, uint32_t rows, uint32_t vocabulary, const void* logits,
                                               uint64_t row_stride, const int32_t* tokens, const float* lse, const float* entropy,
                                               const float* d_logprob, const float* d_entropy, void* d_logits,
                                               uint64_t d_row_stride, uint32_t* device_status, void* hip_stream)
{
    if (!lp_sizes_ok(dtype, rows, vocabulary) || !logits || !tokens || !lse || !d_logprob || !d_logits || !device_status ||
        (d_entropy && !entropy) || (rows > 1 && d_row_stride < vocabulary) || !aligned(logits, bytes_of(dtype)) || !aligned(d_logits, bytes_of(dtype)))
        return STALLOC_ERR_INVALID_ARG;
    const uint32_t chunks = (vocabulary + kLpChunk - 1) / kLpChunk;
    if ((uint64_t)rows * chunks > 0x7fffffffu) return STALLOC_ERR_TOO_LARGE;
    const LogprobBackwardArgs a = {rows, vocabulary, chunks, logits, row_stride, tokens, lse, entropy, d_logprob, d_entropy, d_logits, d_row_stride, device_status};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(lp_backward<decltype(t)>, dim3(rows * chunks), dim3(kLpThreads), 0, stream, a); });
    return launched();
}
