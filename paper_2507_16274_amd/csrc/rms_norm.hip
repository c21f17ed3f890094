// stalloc_rms_norm, stalloc_rms_norm_backward: root-mean-square norm of every row behind the addition of the residual,
//
//     s = round(x + r),   rstd = 1 / sqrt(mean(s^2) + eps),   y = s rstd w,
//     dx = rstd (g - s rstd^2 mean(g s)) + ds   with g = w dy,   dw = sum over rows of dy s rstd.
//
// Both are bound by device memory: a handful of operations per number.  A team of threads, a wave for up to 1024 columns and a workgroup of as many waves as
// the row needs beyond, keeps a whole row in registers between its two looks at it (the sum, then the scaled output), so every input is
// read once and every output written once.  Eight neighbouring numbers belong to a thread: 16-byte accesses, and 128 columns -- what
// one 8-bit scale covers -- are one DPP row of 16 lanes.  8192 rows of 8192 in 16 bits with the output in 8 bits: 86 us, 5.5 TB/s; both passes of 8192 x 5120: 126 us,
// 5.3 TB/s (a large copy: 5.1).
#include "numbers.h"

namespace stalloc {

constexpr float kE4m3Max = 448.f;
constexpr float kLeastScale = 1.1754943508222875e-38f;      // 2^-126: its reciprocal is finite

struct NormArgs {
    uint32_t rows, width;
    const void* x;
    uint64_t x_stride;
    const void* residual;
    uint64_t residual_stride;
    const void* weight;
    float eps;
    void* sum;
    void* y;
    uint8_t* q;
    float* scales;
    float* rstd;
};

// Sum over a team, in all of its threads: a wave (kWaveTeam) or the workgroup.  `part`: one word per wave, not in use.
template <bool kWaveTeam> __device__ __forceinline__ float team_sum(float v, float* part)
{
    v = wave_sum(v);
    if (kWaveTeam) return v;
    if (lane_id() == 0) part[wave_id()] = v;
    __syncthreads();
    float total = 0.f;
    for (uint32_t i = 0; i < blockDim.x / kWave; ++i) total += part[i];
    return total;
}

// The output in 8 bits of eight numbers: the 16 lanes of a DPP row hold 128 columns (lanes past the row's end hold zeros).
// The scale comes from the largest magnitude; compared as bits, so that a NaN counts as larger than everything.
__device__ __forceinline__ void store_eight_bits(f32x8 y, uint32_t row, uint32_t width, uint32_t col, uint8_t* q, float* scales)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = umax(most, as_bits(y[i]) & 0x7fffffffu);
    most = row_max(most);
    float scale = fmaxf(as_float(most), kE4m3Max * kLeastScale) / kE4m3Max;
    if (most >= 0x7f800000u) scale = as_float(0x7fc00000u);
    // y / scale rounded as a division is (Markstein's correction of y times the rounded reciprocal): numbers half way between two of the 8-bit ones are common, since
    // sums and weights have few bits, and two roundings would send some of them the wrong way.
    const float inverse = 1.f / scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = y[i] * inverse;
        y[i] = __builtin_fmaf(-__builtin_fmaf(v, scale, -y[i]), inverse, v);        // (signs as they are: a -0 stays one)
    }
    if (col >= width) return;
    uint32_t word[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        word[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], v, true);
    }
    uint8_t* at = q + (uint64_t)row * width + col;
    if (col + 8 <= width) __builtin_memcpy(at, word, 8);
    else for (uint32_t i = 0; col + i < width; ++i) at[i] = (uint8_t)(word[i / 4] >> (8 * (i & 3)));
    if ((lane_id() & 15) == 0) scales[(uint64_t)row * ((width + 127) / 128) + col / 128] = scale;
}

template <typename T, bool kOnce = false> __device__ __forceinline__ f32x8 add_and_keep(const NormArgs& a, uint32_t row, uint32_t col)
{
    const int n = (int)(a.width - col);
    f32x8 s = load_some_once<kOnce>((const T*)a.x + row * a.x_stride + col, n, 0.f);
    if (a.residual) {
        s += load_some_once<kOnce>((const T*)a.residual + row * a.residual_stride + col, n, 0.f);
        s = __builtin_convertvector(__builtin_convertvector(s, typename Vec<T>::x8), f32x8);
    }
    if (a.sum) store_some((T*)a.sum + (uint64_t)row * a.width + col, n, s);
    return s;
}

__device__ __forceinline__ float square(f32x8 s)
{
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = __builtin_fmaf(s[i], s[i], v);
    return v;
}

template <typename T> __device__ __forceinline__ void emit(const NormArgs& a, uint32_t row, uint32_t col, f32x8 s, float rstd)
{
    const int n = (int)a.width - (int)col;
    f32x8 w = {};
    if (n > 0) w = load_some((const T*)a.weight + col, n, 0.f);
    const f32x8 y = s * rstd * w;
    if (a.y && n > 0) store_some((T*)a.y + (uint64_t)row * a.width + col, n, y);
    if (a.q) store_eight_bits(y, row, a.width, col, a.q, a.scales);
}

// One team per row, kGroups groups of 8 numbers per thread.
//
// kOnce (here and in the backward kernel): inputs go past the caches.  For tensors of 64 MiB and more, four of which a call moves, more than the last cache holds: 8192 rows of
// 8192 in 16 bits with the output in 8 bits, call after call on the same tensors, 87 us without and 76 with it (on other tensors each time 86 and 85), a training pass of
// 8192 x 5120 131 and 121 (132 and 125).  Smaller ones are read faster through the caches (4096 x 4096: 21 us, 24 past them).  Stores past the caches change nothing.
template <typename T, bool kOnce, bool kWaveTeam, int kGroups> __global__ void __launch_bounds__(kWaveTeam ? 256 : 1024) norm_rows(NormArgs a)
{
    __shared__ float part[1024 / kWave];
    const uint32_t team = kWaveTeam ? kWave : blockDim.x;
    const uint32_t row = kWaveTeam ? blockIdx.x * 4 + wave_id() : blockIdx.x, t = kWaveTeam ? lane_id() : threadIdx.x;
    if (row >= a.rows) return;                               // (a whole wave; a workgroup that is a team has a row)
    f32x8 s[kGroups];
    float total = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t col = (g * team + t) * 8;
        s[g] = f32x8{};
        if (col < a.width) s[g] = add_and_keep<T, kOnce>(a, row, col);
        total += square(s[g]);
    }
    const float rstd = 1.f / sqrtf(team_sum<kWaveTeam>(total, part) / (float)a.width + a.eps);
    if (t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) emit<T>(a, row, (g * team + t) * 8, s[g], rstd);
}

// Rows too wide for registers: the second look is at what the first one kept (or at x, where there is no residual).
template <typename T> __global__ void __launch_bounds__(1024) norm_wide(NormArgs a)
{
    __shared__ float part[1024 / kWave];
    const uint32_t row = blockIdx.x;
    float total = 0.f;
    for (uint64_t col = threadIdx.x * 8; col < a.width; col += 8192) total += square(add_and_keep<T>(a, row, (uint32_t)col));
    const float rstd = 1.f / sqrtf(team_sum<false>(total, part) / (float)a.width + a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    const T* kept = a.sum ? (const T*)a.sum + (uint64_t)row * a.width : (const T*)a.x + row * a.x_stride;
    for (uint64_t base = 0; base < a.width; base += 8192) {  // (all lanes stay: 128 columns are reduced over 16 of them)
        const uint64_t col = base + threadIdx.x * 8;
        const int64_t n = (int64_t)a.width - (int64_t)col;
        f32x8 s = {};
        if (n > 0) s = load_some(kept + col, n > 8 ? 8 : (int)n, 0.f);
        emit<T>(a, row, n > 0 ? (uint32_t)col : a.width, s, rstd);
    }
}

struct NormBackwardArgs {
    uint32_t rows, width;
    const void* d_y;
    uint64_t d_y_stride;
    const void* sum;
    const void* weight;
    const float* rstd;
    const void* d_sum;
    void* dx;
    float* part;                                             // [teams][width]: sums of d_y * sum * rstd over a team's rows
};

template <typename T> __device__ __forceinline__ void emit_dx(const NormBackwardArgs& a, uint32_t row, uint32_t col, f32x8 g, f32x8 s, f32x8 d_sum, float r, float c)
{
    store_some((T*)a.dx + (uint64_t)row * a.width + col, (int)(a.width - col), r * (g - s * (r * r * c)) + d_sum);
}

// Every team walks over rows of its own; the thread's columns stay the same, so the weight and the sums of dw are in registers.  The next row is on its way,
// in the type it has in memory, while this one's sum goes round: two teams a CU are enough then, and leave half the
// sums to add up that four would (8192 rows of 5120: 138 us without that and 768 teams, 66 with it).
// kAhead: whether there are registers for that (not with 1024 threads).
template <typename T, bool kOnce, bool kWaveTeam, int kGroups, int kThreads, bool kAhead> __global__ void __launch_bounds__(kThreads) norm_backward_rows(NormBackwardArgs a)
{
    __shared__ float part[2][1024 / kWave];
    using Packed = typename Vec<T>::x8;
    const uint32_t size = kWaveTeam ? kWave : blockDim.x, t = kWaveTeam ? lane_id() : threadIdx.x;
    const uint32_t team = kWaveTeam ? blockIdx.x * 4 + wave_id() : blockIdx.x, teams = kWaveTeam ? gridDim.x * 4 : gridDim.x;
    const auto wide = [](Packed v) { return __builtin_convertvector(v, f32x8); };
    f32x8 w[kGroups], dw[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t col = (g * size + t) * 8;
        dw[g] = w[g] = f32x8{};
        if (col < a.width) w[g] = load_some((const T*)a.weight + col, (int)(a.width - col), 0.f);
    }
    Packed dy[kGroups], s[kGroups], ds[kGroups];
    float r = 0.f;
    const auto fetch = [&](uint32_t row) {
        r = a.rstd[row];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const uint32_t col = (g * size + t) * 8;
            const int n = (int)a.width - (int)col;
            const uint64_t at = (uint64_t)row * a.width + col;
            dy[g] = s[g] = ds[g] = Packed{};
            if (n <= 0) continue;
            dy[g] = packed_some_once<kOnce>((const T*)a.d_y + row * a.d_y_stride + col, n);
            s[g] = packed_some_once<kOnce>((const T*)a.sum + at, n);
            if (a.d_sum) ds[g] = packed_some_once<kOnce>((const T*)a.d_sum + at, n);
        }
    };
    if (kAhead && team < a.rows) fetch(team);
    uint32_t turn = 0;
    for (uint32_t row = team; row < a.rows; row += teams, turn ^= 1) {
        if (!kAhead) fetch(row);
        Packed dy_now[kGroups], s_now[kGroups], ds_now[kGroups];
        const float r_now = r;
        float total = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            dy_now[g] = dy[g];
            s_now[g] = s[g];
            ds_now[g] = ds[g];
            total += dot(wide(dy[g]) * w[g], wide(s[g]));
        }
        if (kAhead && row + teams < a.rows) fetch(row + teams);        // (dx may lie in place of d_y or d_sum: in this row's, never in the next one's)
        const float c = team_sum<kWaveTeam>(total, part[turn]) / (float)a.width;   // (two words in turn: one barrier a row)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const uint32_t col = (g * size + t) * 8;
            const f32x8 y = wide(dy_now[g]), x = wide(s_now[g]);
            dw[g] += y * x * r_now;
            if (col < a.width) emit_dx<T>(a, row, col, y * w[g], x, wide(ds_now[g]), r_now, c);
        }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t col = (g * size + t) * 8;
        if (col < a.width) store_some(a.part + (uint64_t)team * a.width + col, (int)(a.width - col), dw[g]);
    }
}

template <typename T> __global__ void __launch_bounds__(1024) norm_backward_wide(NormBackwardArgs a)
{
    __shared__ float part[1024 / kWave];
    const uint32_t row = blockIdx.x;
    const T* dy = (const T*)a.d_y + row * a.d_y_stride;
    const T* s = (const T*)a.sum + (uint64_t)row * a.width;
    const T* w = (const T*)a.weight;
    const float r = a.rstd[row];
    float total = 0.f;
    for (uint64_t col = threadIdx.x * 8; col < a.width; col += 8192) {
        const int n = (int)(a.width - col);
        total += dot(load_some(dy + col, n, 0.f) * load_some(w + col, n, 0.f), load_some(s + col, n, 0.f));
    }
    const float c = team_sum<false>(total, part) / (float)a.width;
    for (uint64_t col = threadIdx.x * 8; col < a.width; col += 8192) {
        const int n = (int)(a.width - col);
        f32x8 through = {};
        if (a.d_sum) through = load_some((const T*)a.d_sum + (uint64_t)row * a.width + col, n, 0.f);
        emit_dx<T>(a, row, (uint32_t)col, load_some(dy + col, n, 0.f) * load_some(w + col, n, 0.f), load_some(s + col, n, 0.f), through, r, c);
    }
}

// dw of wide rows, before dx is written (dx may be d_y): a workgroup takes 2048 columns and every gridDim.y-th row.
template <typename T> __global__ void __launch_bounds__(256) norm_dweight_wide(NormBackwardArgs a)
{
    const uint64_t col = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= a.width) return;
    const int n = (int)(a.width - col);
    f32x8 dw = {};
    for (uint32_t row = blockIdx.y; row < a.rows; row += gridDim.y)
        dw += load_some((const T*)a.d_y + row * a.d_y_stride + col, n, 0.f) * load_some((const T*)a.sum + (uint64_t)row * a.width + col, n, 0.f) * a.rstd[row];
    store_some(a.part + (uint64_t)blockIdx.y * a.width + col, n, dw);
}

// dweight[c] = sum over the teams, in a fixed order: 64 columns a workgroup at a time, sixteen waves that take a share of the teams each.
__global__ void __launch_bounds__(1024) norm_dweight(const float* __restrict__ part, uint32_t teams, uint32_t width, float* dweight)
{
    __shared__ float sums[16][kWave];
    const uint32_t w = wave_id();
    for (uint32_t first = blockIdx.x * kWave; first < width; first += gridDim.x * kWave) {
        const uint32_t col = first + lane_id();
        float total = 0.f;
        if (col < width) {
            const uint32_t from = (uint32_t)((uint64_t)teams * w / 16), to = (uint32_t)((uint64_t)teams * (w + 1) / 16);
#pragma unroll 8
            for (uint32_t i = from; i < to; ++i) total += part[(uint64_t)i * width + col];
        }
        if (first != blockIdx.x * kWave) __syncthreads();    // (the sums before these have been read)
        sums[w][lane_id()] = total;
        __syncthreads();
        if (w != 0 || col >= width) continue;
#pragma unroll
        for (int i = 1; i < 16; ++i) total += sums[i][lane_id()];
        dweight[col] = total;
    }
}
constexpr uint32_t kMostColumnBlocks = 1u << 16;

constexpr uint32_t kWaveWidth = 1024;                        // rows up to here are a wave's
constexpr uint32_t kWidest = 8 * 1024 * 4, kWidestBackward = 8 * 1024 * 2;         // what a team of 1024 threads keeps in registers

// How a row is shared out: groups of 8 numbers a thread (two, four where two would take more than 1024 threads), and the threads of a workgroup.
struct NormShape {
    uint32_t groups, threads;
};
inline NormShape norm_shape(uint32_t width)
{
    if (width <= kWaveWidth) return {width <= 512 ? 1u : 2u, 256};
    const uint32_t groups = width <= 16384 ? 2 : 4, threads = (width + 8 * groups - 1) / (8 * groups);
    return {groups, (threads + kWave - 1) / kWave * kWave};
}

// Teams of the backward kernel, each with a row of partial sums: eight waves a CU as teams of one wave, else two teams a CU.
inline uint32_t teams_of(uint32_t rows, uint32_t width)
{
    if (width > kWidestBackward) return umin_host(rows, 64);
    if (width <= kWaveWidth) return (umin_host(rows, 2048) + 3) / 4 * 4;
    return umin_host(rows, 512);
}

}  // namespace stalloc

using namespace stalloc;

namespace {

bool read_once(uint32_t dtype, uint32_t rows, uint32_t width) { return (uint64_t)rows * width * bytes_of(dtype) >= (64u << 20); }

// Rows a launch can take, `threads` to each (a multiple of four: waves that are teams come by fours).
uint32_t most_rows(uint32_t threads) { return (uint32_t)(kMostThreads / threads) / 4 * 4; }

// The arguments for rows first .. of a call.
template <typename T> NormArgs rows_from(NormArgs a, uint64_t first, uint32_t rows)
{
    a.rows = rows;
    a.x = (const T*)a.x + first * a.x_stride;
    if (a.residual) a.residual = (const T*)a.residual + first * a.residual_stride;
    if (a.sum) a.sum = (T*)a.sum + first * a.width;
    if (a.y) a.y = (T*)a.y + first * a.width;
    if (a.q) a.q += first * a.width;
    if (a.scales) a.scales += first * ((a.width + 127) / 128);
    a.rstd += first;
    return a;
}
template <typename T> NormBackwardArgs rows_from(NormBackwardArgs a, uint64_t first, uint32_t rows)
{
    a.rows = rows;
    a.d_y = (const T*)a.d_y + first * a.d_y_stride;
    a.sum = (const T*)a.sum + first * a.width;
    a.rstd += first;
    if (a.d_sum) a.d_sum = (const T*)a.d_sum + first * a.width;
    a.dx = (T*)a.dx + first * a.width;
    return a;
}

template <typename T, bool kOnce> void launch_norm_part(const NormArgs& a, hipStream_t stream)
{
    const NormShape shape = norm_shape(a.width);
    const auto one = [&](auto kernel, uint32_t blocks, uint32_t threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a); };
    if (a.width > kWidest) one(norm_wide<T>, a.rows, 1024);
    else if (a.width <= kWaveWidth && shape.groups == 1) one(norm_rows<T, kOnce, true, 1>, (a.rows - 1) / 4 + 1, 256);
    else if (a.width <= kWaveWidth) one(norm_rows<T, kOnce, true, 2>, (a.rows - 1) / 4 + 1, 256);
    else if (shape.groups == 2) one(norm_rows<T, kOnce, false, 2>, a.rows, shape.threads);
    else one(norm_rows<T, kOnce, false, 4>, a.rows, shape.threads);
}

template <typename T, bool kOnce> void launch_norm(const NormArgs& a, hipStream_t stream)
{
    const uint32_t most = most_rows(a.width > kWidest ? 1024 : a.width <= kWaveWidth ? kWave : norm_shape(a.width).threads);
    for (uint64_t first = 0; first < a.rows; first += most) launch_norm_part<T, kOnce>(rows_from<T>(a, first, umin_host(most, a.rows - (uint32_t)first)), stream);
}

template <typename T, bool kOnce> void launch_norm_backward(const NormBackwardArgs& a, uint32_t teams, hipStream_t stream)
{
    const NormShape shape = norm_shape(a.width);
    const auto one = [&](auto kernel, uint32_t blocks, uint32_t threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a); };
    if (a.width > kWidestBackward) {
        hipLaunchKernelGGL(norm_dweight_wide<T>, dim3((a.width + 2047) / 2048, teams), dim3(256), 0, stream, a);
        for (uint64_t first = 0; first < a.rows; first += most_rows(1024)) {
            const NormBackwardArgs part = rows_from<T>(a, first, umin_host(most_rows(1024), a.rows - (uint32_t)first));
            hipLaunchKernelGGL(norm_backward_wide<T>, dim3(part.rows), dim3(1024), 0, stream, part);
        }
    } else if (a.width <= kWaveWidth && shape.groups == 1) one(norm_backward_rows<T, kOnce, true, 1, 256, true>, teams / 4, 256);
    else if (a.width <= kWaveWidth) one(norm_backward_rows<T, kOnce, true, 2, 256, true>, teams / 4, 256);
    else if (shape.threads <= 512) one(norm_backward_rows<T, kOnce, false, 2, 512, true>, teams, shape.threads);
    else one(norm_backward_rows<T, kOnce, false, 2, 1024, false>, teams, shape.threads);
}

bool norm_sizes_ok(uint32_t dtype, uint32_t rows, uint32_t width)
{
    return dtype <= STALLOC_F16 && rows >= 1 && rows < 0x80000000u && width >= 1 && width < 0x7ffff000u;
}

// Whether `out`, rows of `width`, takes the place of rows that lie otherwise: some would be written before they are read.
bool misplaced(const void* out, const void* in, uint64_t stride, uint32_t rows, uint32_t width) { return out && out == in && rows > 1 && stride != width; }

}  // namespace

extern "C" int stalloc_rms_norm(uint32_t dtype, uint32_t rows, uint32_t width, const void* x, uint64_t x_stride, const void* residual,
                                uint64_t residual_stride, const void* weight, float eps, void* sum, void* y, uint8_t* q, float* scales,
                                float* rstd, void* hip_stream)
{
    if (!norm_sizes_ok(dtype, rows, width) || !x || !weight || !rstd || !(eps >= 0.f) || (residual && !sum) || (!y && !q) || (!q) != (!scales))
        return STALLOC_ERR_INVALID_ARG;
    const size_t size = bytes_of(dtype);
    if (!aligned(x, size) || !aligned(residual, size) || !aligned(weight, size) || !aligned(sum, size) || !aligned(y, size)) return STALLOC_ERR_INVALID_ARG;
    if (misplaced(sum, x, x_stride, rows, width) || misplaced(sum, residual, residual_stride, rows, width)) return STALLOC_ERR_INVALID_ARG;
    const NormArgs a = {rows, width, x, x_stride, residual, residual_stride, weight, eps, sum, y, q, scales, rstd};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    begin_launches();
    with_type(dtype, [&](auto t) {
        if (read_once(dtype, rows, width)) launch_norm<decltype(t), true>(a, stream);
        else launch_norm<decltype(t), false>(a, stream);
    });
    return launched();
}

extern "C" int stalloc_rms_norm_backward(uint32_t dtype, uint32_t rows, uint32_t width, const void* d_y, uint64_t d_y_stride,
                                         const void* sum, const void* weight, const float* rstd, const void* d_sum, void* dx,
                                         float* dweight, void* workspace, size_t* workspace_bytes, void* hip_stream)
{
    if (!norm_sizes_ok(dtype, rows, width) || !workspace_bytes) return STALLOC_ERR_INVALID_ARG;
    const uint32_t teams = teams_of(rows, width);
    Carver cv(workspace);
    float* part = cv.take<float>((size_t)teams * width);
    if (!workspace) { *workspace_bytes = cv.used; return STALLOC_OK; }
    if (!d_y || !sum || !weight || !rstd || !dx || !dweight || *workspace_bytes < cv.used || !aligned(workspace, kAlign)) return STALLOC_ERR_INVALID_ARG;
    const size_t size = bytes_of(dtype);
    if (!aligned(d_y, size) || !aligned(sum, size) || !aligned(weight, size) || !aligned(d_sum, size) || !aligned(dx, size)) return STALLOC_ERR_INVALID_ARG;
    if (misplaced(dx, d_y, d_y_stride, rows, width)) return STALLOC_ERR_INVALID_ARG;
    const NormBackwardArgs a = {rows, width, d_y, d_y_stride, sum, weight, rstd, d_sum, dx, part};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    begin_launches();
    with_type(dtype, [&](auto t) {
        if (read_once(dtype, rows, width)) launch_norm_backward<decltype(t), true>(a, teams, stream);
        else launch_norm_backward<decltype(t), false>(a, teams, stream);
    });
    hipLaunchKernelGGL(norm_dweight, dim3(umin_host((width + kWave - 1) / kWave, kMostColumnBlocks)), dim3(1024), 0, stream, part, teams, width, dweight);
    return launched();
}
