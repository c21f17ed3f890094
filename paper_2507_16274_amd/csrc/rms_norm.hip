// stalloc_rms_norm, stalloc_rms_norm_backward: root-mean-square norm of every row behind the addition of the residual,
//
//     s = round(x + r),   rstd = 1 / sqrt(mean(s^2) + eps),   y = s rstd w,
//     dx = rstd (g - s rstd^2 mean(g s)) + ds   with g = w dy,   dw = sum over rows of dy s rstd.
//
// Both are bound by device memory: a handful of operations per number.  A team of 64, 256 or 1024 threads keeps a whole
// row in registers between its two looks at it (the sum, then the scaled output), so every input is read once and every
// output written once.  Eight neighbouring numbers belong to a thread: 16-byte accesses, and 128 columns -- what
// one 8-bit scale covers -- are one DPP row of 16 lanes.
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

// Sum over the kTeam threads of a team (whole waves), in all of them.  `part`: one word per wave, not in use.
template <int kTeam> __device__ __forceinline__ float team_sum(float v, float* part)
{
    v = wave_sum(v);
    if (kTeam == kWave) return v;
    constexpr int kWaves = kTeam / kWave;
    if (lane_id() == 0) part[wave_id()] = v;
    __syncthreads();
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) total += part[i];      // (256 and 1024 threads are a workgroup: one team)
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
    const float inverse = 1.f / scale;
    if (col >= width) return;
    uint32_t word[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i] * inverse, y[4 * i + 1] * inverse, 0, false);
        word[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2] * inverse, y[4 * i + 3] * inverse, v, true);
    }
    uint8_t* at = q + (uint64_t)row * width + col;
    if (col + 8 <= width) __builtin_memcpy(at, word, 8);
    else for (uint32_t i = 0; col + i < width; ++i) at[i] = (uint8_t)(word[i / 4] >> (8 * (i & 3)));
    if ((lane_id() & 15) == 0) scales[(uint64_t)row * ((width + 127) / 128) + col / 128] = scale;
}

template <typename T> __device__ __forceinline__ f32x8 add_and_keep(const NormArgs& a, uint32_t row, uint32_t col)
{
    const int n = (int)(a.width - col);
    f32x8 s = load_some((const T*)a.x + row * a.x_stride + col, n, 0.f);
    if (a.residual) {
        s += load_some((const T*)a.residual + row * a.residual_stride + col, n, 0.f);
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

// One team per row, kGroups groups of 8 numbers per thread: width <= 8 * kTeam * kGroups.
template <typename T, int kTeam, int kGroups>
__global__ void __launch_bounds__(kTeam < 256 ? 256 : kTeam) norm_rows(NormArgs a)
{
    __shared__ float part[kTeam / kWave];
    constexpr int kTeams = kTeam < 256 ? 256 / kTeam : 1;
    const uint32_t row = blockIdx.x * kTeams + threadIdx.x / kTeam, t = threadIdx.x % kTeam;
    if (row >= a.rows) return;                               // (a whole wave; teams of more than one wave have one row a workgroup)
    f32x8 s[kGroups];
    float total = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t col = (g * kTeam + t) * 8;
        s[g] = f32x8{};
        if (col < a.width) s[g] = add_and_keep<T>(a, row, col);
        total += square(s[g]);
    }
    const float rstd = 1.f / sqrtf(team_sum<kTeam>(total, part) / (float)a.width + a.eps);
    if (t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) emit<T>(a, row, (g * kTeam + t) * 8, s[g], rstd);
}

// Rows too wide for registers: the second look is at what the first one kept (or at x, where there is no residual).
template <typename T> __global__ void __launch_bounds__(1024) norm_wide(NormArgs a)
{
    __shared__ float part[1024 / kWave];
    const uint32_t row = blockIdx.x;
    float total = 0.f;
    for (uint64_t col = threadIdx.x * 8; col < a.width; col += 8192) total += square(add_and_keep<T>(a, row, (uint32_t)col));
    const float rstd = 1.f / sqrtf(team_sum<1024>(total, part) / (float)a.width + a.eps);
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

__device__ __forceinline__ float dot(f32x8 a, f32x8 b)
{
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = __builtin_fmaf(a[i], b[i], v);
    return v;
}

template <typename T> __device__ __forceinline__ void emit_dx(const NormBackwardArgs& a, uint32_t row, uint32_t col, f32x8 g, f32x8 s, float r, float c)
{
    const int n = (int)(a.width - col);
    f32x8 d = r * (g - s * (r * r * c));
    const uint64_t at = (uint64_t)row * a.width + col;
    if (a.d_sum) d += load_some((const T*)a.d_sum + at, n, 0.f);
    store_some((T*)a.dx + at, n, d);
}

// Every team walks over rows of its own; the thread's columns stay the same, so the weight and the sums of dw are in registers.
template <typename T, int kTeam, int kGroups>
__global__ void __launch_bounds__(kTeam < 256 ? 256 : kTeam) norm_backward_rows(NormBackwardArgs a)
{
    __shared__ float part[2][kTeam / kWave];
    constexpr int kTeams = kTeam < 256 ? 256 / kTeam : 1;
    const uint32_t team = blockIdx.x * kTeams + threadIdx.x / kTeam, t = threadIdx.x % kTeam, teams = gridDim.x * kTeams;
    f32x8 w[kGroups], dw[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t col = (g * kTeam + t) * 8;
        dw[g] = w[g] = f32x8{};
        if (col < a.width) w[g] = load_some((const T*)a.weight + col, (int)(a.width - col), 0.f);
    }
    uint32_t turn = 0;
    for (uint32_t row = team; row < a.rows; row += teams, turn ^= 1) {
        f32x8 dy[kGroups], s[kGroups];
        float total = 0.f;
        const float r = a.rstd[row];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const uint32_t col = (g * kTeam + t) * 8;
            dy[g] = s[g] = f32x8{};
            if (col < a.width) {
                const int n = (int)(a.width - col);
                dy[g] = load_some((const T*)a.d_y + row * a.d_y_stride + col, n, 0.f);
                s[g] = load_some((const T*)a.sum + (uint64_t)row * a.width + col, n, 0.f);
            }
            total += dot(dy[g] * w[g], s[g]);
        }
        const float c = team_sum<kTeam>(total, part[turn]) / (float)a.width;   // (two words in turn: one barrier a row)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const uint32_t col = (g * kTeam + t) * 8;
            dw[g] += dy[g] * s[g] * r;
            if (col < a.width) emit_dx<T>(a, row, col, dy[g] * w[g], s[g], r, c);
        }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t col = (g * kTeam + t) * 8;
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
    const float c = team_sum<1024>(total, part) / (float)a.width;
    for (uint64_t col = threadIdx.x * 8; col < a.width; col += 8192) {
        const int n = (int)(a.width - col);
        emit_dx<T>(a, row, (uint32_t)col, load_some(dy + col, n, 0.f) * load_some(w + col, n, 0.f), load_some(s + col, n, 0.f), r, c);
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

// dweight[c] = sum over the teams, in their order: 64 columns a workgroup, four waves that take a quarter of the teams each.
__global__ void __launch_bounds__(256) norm_dweight(const float* __restrict__ part, uint32_t teams, uint32_t width, float* dweight)
{
    __shared__ float sums[4][kWave];
    const uint32_t col = blockIdx.x * kWave + lane_id(), w = wave_id();
    float total = 0.f;
    if (col < width) {
        const uint32_t from = (uint32_t)((uint64_t)teams * w / 4), to = (uint32_t)((uint64_t)teams * (w + 1) / 4);
#pragma unroll 8
        for (uint32_t i = from; i < to; ++i) total += part[(uint64_t)i * width + col];
    }
    sums[w][lane_id()] = total;
    __syncthreads();
    if (w == 0 && col < width) dweight[col] = (sums[0][lane_id()] + sums[1][lane_id()]) + (sums[2][lane_id()] + sums[3][lane_id()]);
}

constexpr uint32_t kWidest = 8 * 1024 * 4;                   // what a team of 1024 threads keeps in registers

inline uint32_t team_of(uint32_t width) { return width <= 1024 ? 64 : width <= 8192 ? 256 : 1024; }

// Teams of the backward kernel, each with a row of partial sums: enough for the waves that fill the chip.
inline uint32_t teams_of(uint32_t rows, uint32_t width)
{
    if (width > kWidest) return umin_host(rows, 64);
    const uint32_t team = team_of(width), most = team == 64 ? 2048 : team == 256 ? 768 : 256;
    const uint32_t teams = umin_host(rows, most);
    return team == 64 ? (teams + 3) / 4 * 4 : teams;
}

}  // namespace stalloc

using namespace stalloc;

namespace {

template <typename T> void launch_norm(const NormArgs& a, hipStream_t stream)
{
    const uint32_t groups = (uint32_t)(((uint64_t)a.width + 8 * team_of(a.width) - 1) / (8 * team_of(a.width)));
    const auto one = [&](auto kernel, uint32_t blocks, uint32_t threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a); };
    if (a.width > kWidest) one(norm_wide<T>, a.rows, 1024);
    else if (team_of(a.width) == 64 && groups == 1) one(norm_rows<T, 64, 1>, (a.rows - 1) / 4 + 1, 256);
    else if (team_of(a.width) == 64) one(norm_rows<T, 64, 2>, (a.rows - 1) / 4 + 1, 256);
    else if (team_of(a.width) == 256 && groups == 1) one(norm_rows<T, 256, 1>, a.rows, 256);
    else if (team_of(a.width) == 256 && groups == 2) one(norm_rows<T, 256, 2>, a.rows, 256);
    else if (team_of(a.width) == 256) one(norm_rows<T, 256, 4>, a.rows, 256);
    else if (groups <= 2) one(norm_rows<T, 1024, 2>, a.rows, 1024);
    else one(norm_rows<T, 1024, 4>, a.rows, 1024);
}

template <typename T> void launch_norm_backward(const NormBackwardArgs& a, uint32_t teams, hipStream_t stream)
{
    const uint32_t groups = (uint32_t)(((uint64_t)a.width + 8 * team_of(a.width) - 1) / (8 * team_of(a.width)));
    const auto one = [&](auto kernel, uint32_t blocks, uint32_t threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a); };
    if (a.width > kWidest) {
        hipLaunchKernelGGL(norm_dweight_wide<T>, dim3((a.width + 2047) / 2048, teams), dim3(256), 0, stream, a);
        one(norm_backward_wide<T>, a.rows, 1024);
    } else if (team_of(a.width) == 64 && groups == 1) one(norm_backward_rows<T, 64, 1>, teams / 4, 256);
    else if (team_of(a.width) == 64) one(norm_backward_rows<T, 64, 2>, teams / 4, 256);
    else if (team_of(a.width) == 256 && groups == 1) one(norm_backward_rows<T, 256, 1>, teams, 256);
    else if (team_of(a.width) == 256 && groups == 2) one(norm_backward_rows<T, 256, 2>, teams, 256);
    else if (team_of(a.width) == 256) one(norm_backward_rows<T, 256, 4>, teams, 256);
    else if (groups <= 2) one(norm_backward_rows<T, 1024, 2>, teams, 1024);
    else one(norm_backward_rows<T, 1024, 4>, teams, 1024);
}

bool norm_sizes_ok(uint32_t dtype, uint32_t rows, uint32_t width)
{
    return dtype <= STALLOC_F16 && rows >= 1 && rows < 0x80000000u && width >= 1 && width < 0x7ffff000u;
}

}  // namespace

extern "C" int stalloc_rms_norm(uint32_t dtype, uint32_t rows, uint32_t width, const void* x, uint64_t x_stride, const void* residual,
                                uint64_t residual_stride, const void* weight, float eps, void* sum, void* y, uint8_t* q, float* scales,
                                float* rstd, void* hip_stream)
{
    if (!norm_sizes_ok(dtype, rows, width) || !x || !weight || !rstd || !(eps >= 0.f) || (residual && !sum) || (!y && !q) || (!q) != (!scales))
        return STALLOC_ERR_INVALID_ARG;
    const size_t size = bytes_of(dtype);
    if (!aligned(x, size) || !aligned(residual, size) || !aligned(weight, size) || !aligned(sum, size) || !aligned(y, size)) return STALLOC_ERR_INVALID_ARG;
    const NormArgs a = {rows, width, x, x_stride, residual, residual_stride, weight, eps, sum, y, q, scales, rstd};
    with_type(dtype, [&](auto t) { launch_norm<decltype(t)>(a, static_cast<hipStream_t>(hip_stream)); });
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
    const NormBackwardArgs a = {rows, width, d_y, d_y_stride, sum, weight, rstd, d_sum, dx, part};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    with_type(dtype, [&](auto t) { launch_norm_backward<decltype(t)>(a, teams, stream); });
    hipLaunchKernelGGL(norm_dweight, dim3((width + kWave - 1) / kWave), dim3(256), 0, stream, part, teams, width, dweight);
    return launched();
}
