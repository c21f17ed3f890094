// stalloc_token_logprobs, stalloc_token_logprobs_backward: the softmax over a vocabulary without its probabilities.
//
//     m = max x,  Z = sum exp(x - m),  A = sum exp(x - m) (x - m):   lse = m + ln Z,  log p_y = x_y - lse,  H = ln Z - A / Z
//     dx_j = g ([j = y] - p_j) - h p_j (ln p_j + H)
//
// One pass over the logits with a running maximum: eight numbers at a time raise m, and Z and A are brought to the new m by
// one factor.  Sums are kept in units of log 2, (x - m) log2(e), for the hardware's exponential.  Few rows are cut
// into parts so that the whole chip reads, and a workgroup per row joins them.
//
// Bound by device memory: 4096 x 131072 in 16 bits, both passes (the logits read twice, their gradient written), 527 us, 6.1 TB/s; 16 x 50257 in 32 bits with 16 alternatives, 15 us, are
// two launches of which half is picking alternatives.
//
// The most likely tokens cost no second pass: a thread remembers which group of eight gave it its maximum (the running maximum
// it needs anyway).  The k-th largest of the 256 maxima bounds the k-th largest number from below, and the numbers that reach it all belong to the
// k threads with the largest maxima: those threads' numbers alone (k 256ths of the part) are looked at again, by whole waves, and what
// reaches the bound, hardly more than k numbers as a rule, is put in order by counting.
#include <math.h>

#include "numbers.h"

namespace stalloc {

constexpr uint32_t kMostTop = 64;
constexpr uint32_t kMostParts = 64;
constexpr int kLpThreads = 256;

// A number and its place as one integer: larger numbers first, then lower places; 0 is below all.  -0 counts as 0, NaN of either sign as larger than infinity: a thread's maximum, which
// passes over NaN, is then never above what the thread holds.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t place)
{
    const uint32_t b = x != x ? 0x7fc00000u : as_bits(x + 0.f);
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

// Over the lanes of a wave, in all of them: to one maximum first, then sums.
__device__ __forceinline__ Softmax join_wave(Softmax s)
{
    float m = s.m;
    m = fmaxf(m, dpp<kDppRowRor8>(kLowest, m));
    m = fmaxf(m, dpp<kDppRowRor4>(kLowest, m));
    m = fmaxf(m, dpp<kDppRowRor2>(kLowest, m));
    m = fmaxf(m, dpp<kDppRowRor1>(kLowest, m));
    m = fmaxf(m, dpp<kDppRowBcast15, 0xa>(kLowest, m));
    m = fmaxf(m, dpp<kDppRowBcast31, 0xc>(kLowest, m));
    rebase(s, as_float(__builtin_amdgcn_readlane(as_bits(m), kWave - 1)));
    s.z = wave_sum(s.z);
    s.a = wave_sum(s.a);
    return s;
}

__device__ __forceinline__ float max_of(f32x8 v) { return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]))); }

__device__ __forceinline__ Softmax with_eight(Softmax s, f32x8 v)
{
    rebase(s, fmaxf(s.m, max_of(v)));
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
    s = join_wave(s);
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

// The row's token and its logit: asked for when a workgroup begins, wanted when it ends.
struct Target {
    int32_t token;
    float logit;
};
template <typename T> __device__ __forceinline__ Target target_of(const LogprobArgs& a, uint32_t row)
{
    Target t = {a.tokens[row], 0.f};
    if (t.token >= (int32_t)a.vocabulary) t.token = -1;
    if (t.token >= 0) t.logit = (float)((const T*)a.logits)[row * a.row_stride + t.token];
    return t;
}

__device__ __forceinline__ void finish_row(const LogprobArgs& a, uint32_t row, const Softmax& s, Target target)
{
    const float ln_z = logf(s.z);                            // (log 0 = -infinity: nothing can occur)
    a.logprob[row] = target.token < 0 ? 0.f : s.z == 0.f ? -INFINITY : (target.logit - s.m) - ln_z;
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

// The key of rank `rank` of the workgroup's part: to the row's outputs, or to the part's list.
__device__ __forceinline__ void put_key(const LogprobArgs& a, uint32_t row, uint32_t rank, uint64_t key, const Softmax& s)
{
    if (a.parts > 1) a.keys[(uint64_t)blockIdx.x * a.top + rank] = key;
    else put_top(a, row, rank, key, s);
}

constexpr uint32_t kMostFound = 1024;

// A workgroup takes one part of one row.
//
// kOnce: logits (and their gradient, in lp_backward) go past the caches.  For tensors of 256 MiB and more, which no cache keeps for whoever reads them
// next: 4096 x 131072 in 16 bits, both passes, 595 us without and 537 with it.  Smaller ones are left to the caches.
template <typename T, bool kOnce> __global__ void __launch_bounds__(kLpThreads) lp_row(LogprobArgs a)
{
    __shared__ Softmax waves[kLpThreads / kWave];
    __shared__ uint64_t best[kLpThreads], rows_best[kLpThreads / 16], list[kMostFound], bound;
    __shared__ uint32_t found[2];
    __shared__ uint8_t first[kLpThreads];
    __shared__ uint32_t words[kLpThreads / kWave];
    if (blockIdx.x == 0) check_tokens(a.tokens, a.rows, a.vocabulary, a.status, words);
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts, t = threadIdx.x;
    const T* x = (const T*)a.logits + row * a.row_stride;
    const uint32_t from = part * a.part_width, to = umin(a.vocabulary, from + a.part_width);   // (the last parts may be empty: from >= to)
    const Target target = target_of<T>(a, row);
    Softmax s = of_nothing();
    float most = -INFINITY;                                  // this thread's maximum, and where it was met first
    uint32_t group = from + t * 8;
    const auto take = [&](uint32_t at, f32x8 v) {
        const float m = max_of(v);
        if (m > most) group = at;
        most = fmaxf(most, m);
        s = with_eight(s, v);
    };
    constexpr uint32_t kStride = kLpThreads * 8;
    uint32_t at = from + t * 8;
    for (; at + kStride + 8 <= to; at += 2 * kStride) {      // two accesses under way: 199 us for 4096 x 131072 in 16 bits with one, 190 with two, 192 with four
        const f32x8 v = load_some_once<kOnce>(x + at, 8, 0.f), w = load_some_once<kOnce>(x + at + kStride, 8, 0.f);
        take(at, v);
        take(at + kStride, w);
    }
    for (; at < to; at += kStride) take(at, load_some_once<kOnce>(x + at, (int)(to - at), -INFINITY));
    if (a.top) best[t] = group < to ? key_of(most, group) : 0;
    s = join_workgroup(s, waves);                            // (behind its barrier the maxima are there as well)
    if (t == 0) {
        if (a.parts > 1) a.part[blockIdx.x] = s;
        else finish_row(a, row, s, target);
    }
    if (!a.top) return;

    // Ranks among the maxima (all different but for threads without numbers, which have 0): the first `top` threads, and their last one's maximum.  For up to
    // 16 only maxima that reach the `top`-th largest of the 16 DPP rows' take part.
    const uint32_t top = a.top, threads = (to > from ? to - from + 7 : 0) / 8;       // threads with numbers
    const uint64_t mine = best[t];
    uint64_t row_best = mine;
    row_best = umax64(row_best, dpp64<kDppRowRor1>(0, row_best));
    row_best = umax64(row_best, dpp64<kDppRowRor2>(0, row_best));
    row_best = umax64(row_best, dpp64<kDppRowRor4>(0, row_best));
    row_best = umax64(row_best, dpp64<kDppRowRor8>(0, row_best));
    if ((t & 15) == 0) rows_best[t / 16] = row_best;
    if (t < 2) found[t] = 0;
    if (t == 0) bound = 1;                                   // (fewer than `top` maxima: all numbers count)
    __syncthreads();
    uint64_t pivot = 1;
    if (top <= kLpThreads / 16) {
        const uint64_t other = rows_best[t & 15];
        uint32_t larger = 0;
#pragma unroll
        for (int i = 0; i < kLpThreads / 16; ++i) larger += rows_best[i] > other;
        const uint64_t at = __ballot(larger == top - 1 && other != 0);
        if (at) pivot = readlane64(other, __builtin_ctzll(at));
    }
    if (mine >= pivot) list[atomicAdd(&found[0], 1u)] = mine;
    __syncthreads();
    if (t < found[0]) {
        const uint64_t k = list[t];
        uint32_t rank = 0;
#pragma unroll 4
        for (uint32_t i = 0; i < found[0]; ++i) rank += list[i] > k;
        if (rank < top) first[rank] = (uint8_t)((place_of(k) - from) / 8 % kLpThreads);
        if (rank == top - 1) bound = k - 7;                  // (the maximum is one of the eight numbers from that place on)
    }
    __syncthreads();
    const uint64_t least = bound;
    for (uint32_t i = wave_id(); i < umin(top, threads); i += kLpThreads / kWave)
        for (uint32_t at = from + (first[i] + lane_id() * kLpThreads) * 8; at < to; at += kWave * kLpThreads * 8) {
            const f32x8 v = load_some(x + at, (int)(to - at), -INFINITY);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint64_t k = key_of(v[j], at + j);
                if (at + j >= to || k < least) continue;
                const uint32_t place = atomicAdd(&found[1], 1u);
                if (place < kMostFound) list[place] = k;
            }
        }
    __syncthreads();
    const uint32_t n = found[1];
    if (n <= kMostFound) {
        for (uint32_t i = t; i < n; i += kLpThreads) {
            const uint64_t k = list[i];
            uint32_t r = 0;
#pragma unroll 4
            for (uint32_t j = 0; j < n; ++j) r += list[j] > k;
            if (r < top) put_key(a, row, r, k, s);
        }
        for (uint32_t i = n + t; i < top; i += kLpThreads) put_key(a, row, i, 0, s);       // (a part shorter than `top`)
        return;
    }
    // More than there is room for (thousands of large numbers in few threads' columns): one after the other, each the largest below the one before.
    uint64_t below = ~0ull;
    for (uint32_t r = 0; r < top; ++r) {
        uint64_t k = 0;
        for (uint32_t at = from + t * 8; at < to; at += kLpThreads * 8) {
            const f32x8 v = load_some(x + at, (int)(to - at), -INFINITY);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint64_t other = key_of(v[j], at + j);
                if (at + j < to && other < below) k = umax64(k, other);
            }
        }
        k = wave_max64(k);
        __syncthreads();
        if (lane_id() == 0) best[wave_id()] = k;
        __syncthreads();
        for (int i = 0; i < kLpThreads / kWave; ++i) k = umax64(k, best[i]);
        if (t == 0) put_key(a, row, r, k, s);
        below = k;
    }
}


// A workgroup joins the parts of a row (at most 64), and picks the row's most likely tokens from theirs, which every part lists in descending
// order: a key's rank is the number of larger keys, counted, or (more than 1024 of them) its place in its own list and, in each other one, the number of
// larger keys, found by halving.
template <typename T> __global__ void __launch_bounds__(kLpThreads) lp_join(LogprobArgs a)
{
    __shared__ uint64_t keys[kMostParts * kMostTop];
    const uint32_t row = blockIdx.x, lane = lane_id(), all = a.parts * a.top;
    for (uint32_t i = threadIdx.x; i < all; i += kLpThreads) keys[i] = a.keys[(uint64_t)row * all + i];
    const Target target = target_of<T>(a, row);
    Softmax s = of_nothing();
    if (lane < a.parts) s = a.part[(uint64_t)row * a.parts + lane];
    s = join_wave(s);
    if (threadIdx.x == 0) finish_row(a, row, s, target);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < all; i += kLpThreads) {
        const uint64_t k = keys[i];
        uint32_t rank = 0;
        if (all <= 1024) {
#pragma unroll 8
            for (uint32_t j = 0; j < all; ++j) rank += keys[j] > k;
        } else {
            const uint32_t part = i / a.top;
            rank = i % a.top;
            for (uint32_t p = 0; p < a.parts && rank < a.top; ++p) {
                if (p == part) continue;
                const uint64_t* list = keys + p * a.top;
                uint32_t lo = 0, hi = a.top;                 // list[0 .. lo) are larger, list[hi ..) are not
                while (lo < hi) {
                    const uint32_t mid = (lo + hi) / 2;
                    if (list[mid] > k) lo = mid + 1;
                    else hi = mid;
                }
                rank += lo;
            }
        }
        if (k && rank < a.top) put_top(a, row, rank, k, s);
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
// Where p is near 1 what is left of 1 - p is as good as lse, half a step of 32 bits of which (5e-7 for an lse of 8 to 16) is all that the backward pass loses; with 32-bit logits
// that is what one sees (d_logits 2e-6 to 3e-6 off, 1e-6 from probabilities that are normalised anew, for which the row would have to be read twice).
// An lse beyond 256 (logits around a type's lowest value, say) says too little in 32 bits: the first workgroup of such a row then
// sums it up again and writes all of it.
template <typename T, bool kOnce> __global__ void __launch_bounds__(kLpThreads) lp_backward(LogprobBackwardArgs a)
{
    __shared__ uint32_t words[kLpThreads / kWave];
    __shared__ Softmax waves[kLpThreads / kWave];
    if (blockIdx.x == 0) check_tokens(a.tokens, a.rows, a.vocabulary, a.status, words);
    const uint32_t row = a.rows - 1 - blockIdx.x / a.chunks;  // last rows first: they are what the forward pass left in the caches
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
            const f32x8 v = load_some_once<kOnce>(x + at, n, -INFINITY);
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
            if (kOnce && n >= 8) store8_once(d + at, out);
            else store_some(d + at, n, out);
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

bool read_once(uint32_t dtype, uint32_t rows, uint32_t vocabulary) { return (uint64_t)rows * vocabulary * bytes_of(dtype) >= (256u << 20); }

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
    begin_launches();
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (read_once(dtype, rows, vocabulary)) hipLaunchKernelGGL((lp_row<T, true>), dim3(rows * shape.parts), dim3(kLpThreads), 0, stream, a);
        else hipLaunchKernelGGL((lp_row<T, false>), dim3(rows * shape.parts), dim3(kLpThreads), 0, stream, a);
        if (shape.parts > 1) hipLaunchKernelGGL(lp_join<T>, dim3(rows), dim3(kLpThreads), 0, stream, a);
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
    if (d_logits == logits && rows > 1 && d_row_stride != row_stride) return STALLOC_ERR_INVALID_ARG;      // (rows would be written that are still to be read)
    const uint32_t chunks = (vocabulary + kLpChunk - 1) / kLpChunk;
    if ((uint64_t)rows * chunks * kLpThreads > kMostThreads) return STALLOC_ERR_TOO_LARGE;
    const LogprobBackwardArgs a = {rows, vocabulary, chunks, logits, row_stride, tokens, lse, entropy, d_logprob, d_entropy, d_logits, d_row_stride, device_status};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    begin_launches();
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (read_once(dtype, rows, vocabulary)) hipLaunchKernelGGL((lp_backward<T, true>), dim3(rows * chunks), dim3(kLpThreads), 0, stream, a);
        else hipLaunchKernelGGL((lp_backward<T, false>), dim3(rows * chunks), dim3(kLpThreads), 0, stream, a);
    });
    return launched();
}
