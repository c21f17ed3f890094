// stalloc_attention: causal attention over packed sequences, scores and weights in registers.
//
//     o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - lse_i),  lse_i = log sum_{j <= i} exp(scale q_i . k_j)
//
// A workgroup of four waves takes 128 rows of one head, a wave 32 of them; keys and values pass through LDS 64 at a time.  A
// wave computes the transposed scores K Q^T (keys as rows), so that a row's scores are in two lanes only: maximum and sum are taken in
// registers, and the weights are, where they lie, the operand of the next product V^T P^T (attention.h).
//
// Bound by the matrix pipe and vector issue together: 32 matrix instructions a wave and tile (1024 cycles with heads of 128) against some 175 vector ones, 32 exponentials among
// them (1100 cycles), of which two waves a SIMD hide most.  One sequence of 8192, 64 heads of 128: 1027 us, 1.07 PFLOP/s, matrix pipe busy 58 % (a product of 16384^3
// reaches 1.37).  Short sequences are bound by the beginnings and ends of workgroups: 23 of them, 8000 tokens, 32 heads of 128: 101 us, 0.57 PFLOP/s.
#include "attention.h"

namespace stalloc {

template <typename T> struct AttentionArgs {
    Heads<T> q, k, v, o;
    float* lse;
    uint32_t* status;
    Work work;
    float* partial;                                          // [parts][heads][tokens][head_dim]: sums of a part, if there are several
    f32x2* part_stats;                                       // [parts][heads][tokens]: largest score and sum of weights of a part
    uint32_t group, head_dim;
    float scale;
};

// Tiles of a part at least: two more kernels' beginnings and ends are about as long as a few tiles.  One sequence of 4096, 4 heads of 128: 72 us in one part, 39 in four.
constexpr uint32_t kLeastSteps = 4;
constexpr int kAttnThreads = 256, kAttnRows = kPieceRows, kAttnKeys = 64, kAttnStages = 2, kAttnTiles = kAttnKeys / 32;

// Weights of the walk by tiles are 2^(scale s - shift), shift = scale m rounded, in one operation; everything that is relative to m is relative to this shift.  Where shift is
// huge, what rounding left of scale m is whole powers of two, and scale m itself may overflow: rows like that (and rows whose scores are all -infinity) are made again, pair by pair, with weights 2^(scale
// (s - m)).
constexpr float kFarScore = 1 << 16;

// scale m, rounded (and not left to an operation behind it, which would make of the difference of two of them what rounding left of one).
__device__ __forceinline__ float shift_of(float m, float scale)
{
#pragma clang fp contract(off)
    return m * scale;
}

// o of a wave's rows over keys from .. to - 1, pair by pair (attention.h).  m, total: their largest scores and the lanes' shares of the sums of weights, which do not depend on what
// other keys stand for; made again where scores are far.
template <typename T, int kD, bool kFull>
__device__ __forceinline__ void rows_again(const AttentionArgs<T>& a, const Piece& p, uint32_t head, uint32_t from, uint32_t to, bool far, float& m, float& total, f32x16 (&o)[kD / 32])
{
    const uint32_t first = p.first + 32 * wave_id(), row = first + (lane_id() & 31), last = p.end - 1, kv = head / a.group;
    const uint32_t behind = umin(to, umin(first + 31, last) + 1);
    const float scale = a.scale * kLog2e;
    V8<T> q[kD / 16];
    load_row<T, kD, kFull>(q, a.q.at(umin(row, last), head), a.head_dim);
#pragma unroll
    for (int d = 0; d < kD / 32; ++d) o[d] = f32x16{};
    if (far) {
        const f32x2 stats = row_stats<T, kD, kFull>(q, a.k.at(0, kv), a.k.token, from, behind, row, scale, a.head_dim);
        m = stats[0];
        total = lane_id() < 32 ? stats[1] : 0.f;
    }
#pragma unroll 1
    for (uint32_t key = from; key < behind; ++key) {
        const float s = dot_row<T, kD, kFull>(q, a.k.at(key, kv), a.head_dim);
        const float w = exp2_fast(far ? (s - m) * scale : __builtin_fmaf(s, scale, -shift_of(m, scale)));
        if (key <= row) add_row<T, kD, kFull>(o, w, a.v.at(key, kv), a.head_dim);
        if (key % 32 == 0 && __all(all_nan(o, a.head_dim))) return;
    }
}

template <typename T, int kD, bool kFull> __global__ void __launch_bounds__(kAttnThreads, kD == 64 ? 4 : 2) attention_rows(AttentionArgs<T> a)
{
    __shared__ __attribute__((aligned(256))) T ring[kAttnStages][2][kAttnKeys * kD];       // keys, values
    if (blockIdx.x == 0 && !a.work.list) check_bounds(a.work.bounds, a.work.sequences, a.work.tokens, a.status);
    const Task task = take_task<kAttnRows, true>(a.work);
    const Piece p = task.piece;
    const uint32_t head = task.head;
    if (p.first >= p.end) return;
    const uint32_t half = lane_id() >> 5, first = p.first + 32 * wave_id(), row = first + (lane_id() & 31);
    const uint32_t parts = a.work.parts, part = task.part;
    const uint64_t part_row = ((uint64_t)part * a.work.heads + head) * a.work.tokens + row;
    if (p.no_keys) {
        if (row < p.end && parts > 1) {
            if (half == 0) a.part_stats[part_row] = f32x2{kNoScore, -1.f};       // (of no row that sees something)
        } else if (row < p.end) {
            const f32x16 zero[kD / 32] = {};
            store_row<T, kD, kFull>(a.o.at(row, head), zero, 0.f, a.head_dim);
            if (half == 0) a.lse[(uint64_t)head * a.work.tokens + row] = -INFINITY;
        }
        return;
    }
    const uint32_t last = p.end - 1, kv = head / a.group;
    const T* k = a.k.at(0, kv);
    const T* v = a.v.at(0, kv);
    const float scale = a.scale * kLog2e, slack = 8.f / scale;
    const Places<kD> places;
    // Running maximum (of unscaled scores; what it begins with is below all that it could be, and finite when it is scaled), the lane's share of the sum.
    float m = -fminf(3e38f, 1.5e38f / scale), total = 0.f;
    f32x16 o[kD / 32] = {};
    // The walk: tiles of keys up to the last row's; this part's share of them.
    const uint32_t all = (umin(p.first + kAttnRows, p.end) - p.begin + kAttnKeys - 1) / kAttnKeys;
    const uint32_t from = p.begin + (uint32_t)((uint64_t)all * part / parts) * kAttnKeys;
    const uint32_t steps = (uint32_t)((uint64_t)all * (part + 1) / parts) - (from - p.begin) / kAttnKeys;
    using Tile = Rows<T, kD, kAttnKeys, kAttnThreads, kFull>;
    const auto fetch = [&](uint32_t step) {
        T (&stage)[2][kAttnKeys * kD] = ring[step % kAttnStages];
        Tile::fetch(stage[0], k, a.k.token, from + step * kAttnKeys, last, a.head_dim);
        Tile::fetch(stage[1], v, a.v.token, from + step * kAttnKeys, last, a.head_dim);
    };
    if (!kFull) clear_lds<sizeof(ring) / 4, kAttnThreads>(ring);
#pragma unroll
    for (uint32_t step = 0; step < kAttnStages - 1; ++step)
        if (step < steps) fetch(step);
    V8<T> q[kD / 16];
    load_row<T, kD, kFull>(q, a.q.at(umin(row, last), head), a.head_dim);
    vector_memory_done();                                    // (q is here before the loop: its loads are not waited for among the tiles')
    for (uint32_t step = 0; step < steps; ++step) {
        const uint32_t key = from + step * kAttnKeys;
        constexpr uint32_t kTile = sizeof(ring[0][0]);
        const uint32_t tile = step % kAttnStages * 2 * kTile, along = kept(tile + places.along), cross = kept(tile + places.cross);
        if (step + kAttnStages - 1 < steps) {
            tiles_landed<2 * Tile::kLoads * (kAttnStages - 2)>();
            fetch(step + kAttnStages - 1);
        } else {
            tiles_landed<0>();
        }
        if (key <= first + 31 && first < p.end) {            // (else none of the wave's rows sees any of these keys, or it has no rows)
            f32x16 s[kAttnTiles] = {};
            products<kAttnTiles * kD / 16, 4, T>([&](int i) { return read_along<T, kD>(ring[0][0], along, i / kAttnTiles, 64 * kD * (i % kAttnTiles)); },
                                                 [&](int i, V8<T> k) { s[i % kAttnTiles] = mma(k, q[i / kAttnTiles], s[i % kAttnTiles]); });
            if (key + kAttnKeys - 1 > first) {
#pragma unroll
                for (int t = 0; t < kAttnTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key + 32 * t + row_of(i, half) > row) s[t][i] = -INFINITY;
            }
            float most = -INFINITY;
#pragma unroll
            for (int t = 0; t < kAttnTiles; ++t)
#pragma unroll
                for (int i = 0; i < 16; i += 8) {
                    const float a0 = max3(s[t][i], s[t][i + 1], s[t][i + 2]), a1 = max3(s[t][i + 3], s[t][i + 4], s[t][i + 5]);
                    most = max3(most, a0, max3(a1, s[t][i + 6], s[t][i + 7]));
                }
            most = fmaxf(most, across(most));
            // The maximum is raised only where weights would pass 2^8 otherwise: sums and results are relative to it all the same.
            if (__any(most > m + slack)) {
                const float raised = fmaxf(m, most), f = exp2_fast(shift_of(m, scale) - shift_of(raised, scale));
                m = raised;
                total *= f;
#pragma unroll
                for (int d = 0; d < kD / 32; ++d) o[d] *= f;
            }
            const float shift = shift_of(m, scale);
            float sums[4] = {total, 0.f, 0.f, 0.f};          // (four chains of additions)
#pragma unroll
            for (int t = 0; t < kAttnTiles; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[t][i] = exp2_fast(__builtin_fmaf(s[t][i], scale, -shift));
                    sums[i % 4] += s[t][i];
                }
            total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            // Weights are rounded to T for the product (half a step of T each, and of alternating sign); their sum is not.
            V8<T> w[2 * kAttnTiles];
#pragma unroll
            for (int t = 0; t < kAttnTiles; ++t) {
                w[2 * t] = operand<T, 0>(s[t]);
                w[2 * t + 1] = operand<T, 1>(s[t]);
            }
            constexpr int kDs = kD / 32;
            products<2 * kAttnTiles * kDs, 4, T>([&](int i) { return read_cross<T, kD>(ring[0][0], cross, i % kDs, kTile + 32 * kD * (i / kDs)); },
                                                 [&](int i, V8<T> v) { o[i % kDs] = mma(v, w[i / kDs], o[i % kDs]); });
        }
    }
    // (A row may see nothing of a part; one that saw a NaN stays as it is.)
    const bool far = __any(fabsf(m * scale) > kFarScore && steps && row >= from && row < p.end && total == total);
    if (far || __any(not_finite(o))) rows_again<T, kD, kFull>(a, p, head, from, from + steps * kAttnKeys, far, m, total, o);
    total += across(total);
    if (row >= p.end) return;
    if (parts > 1) {
        if (half == 0) a.part_stats[part_row] = f32x2{m, total};
        if (steps) store_row<float, kD, kFull>(a.partial + part_row * a.head_dim, o, 1.f, a.head_dim);
        return;
    }
    // (A row whose scores are all -infinity has no weights: 0 / 0.)
    store_row<T, kD, kFull>(a.o.at(row, head), o, 1.f / total, a.head_dim);
    if (half == 0) a.lse[(uint64_t)head * a.work.tokens + row] = __builtin_fmaf(log2f(total), kLn2, m * a.scale);
}

// o and lse from the parts': eight columns of a row a thread.
template <typename T> __global__ void __launch_bounds__(256) attention_join(AttentionArgs<T> a)
{
    const uint32_t pieces = a.head_dim / 8;
    const uint64_t rows = (uint64_t)a.work.heads * a.work.tokens, at = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = at / pieces;
    const uint32_t col = (uint32_t)(at % pieces) * 8;
    if (row >= rows) return;
    const float scale = a.scale * kLog2e;
    float m = kNoScore, total = 0.f;
    for (uint32_t part = 0; part < a.work.parts; ++part) {
        const f32x2 stats = a.part_stats[part * rows + row];
        if (!(stats[1] <= 0.f)) m = fmaxf(m, stats[0]);
    }
    f32x8 o = {};
    for (uint32_t part = 0; part < a.work.parts; ++part) {
        const f32x2 stats = a.part_stats[part * rows + row];
        if (stats[1] <= 0.f) continue;                       // (saw nothing: its sums may not be there)
        const float f = exp2_fast(fabsf(m * scale) > kFarScore ? (stats[0] - m) * scale : shift_of(stats[0], scale) - shift_of(m, scale));
        total += stats[1] * f;
        o += load8(a.partial + (part * rows + row) * a.head_dim + col) * f;
    }
    const uint32_t head = (uint32_t)(row / a.work.tokens), token = (uint32_t)(row % a.work.tokens);
    const bool padding = a.part_stats[row][1] < 0.f;
    store8(a.o.at(token, head) + col, o * (padding ? 0.f : 1.f / total));
    if (col == 0) a.lse[row] = __builtin_fmaf(log2f(total), kLn2, m * a.scale);
}

// All pieces of the batch, those with the longest walks first: counted by length (of their walk, in pieces), placed by count.  One workgroup; a wave takes a
// sequence at a time.  Which of the pieces of one length comes first depends on scheduling, and nothing depends on that.
constexpr int kListThreads = 1024, kListLengths = 1024;

__global__ void __launch_bounds__(kListThreads) attention_list(const uint32_t* __restrict__ bounds, uint32_t sequences, uint32_t tokens, uint32_t pieces, uint4* list,
                                                               uint32_t* status)
{
    __shared__ uint32_t whole[kListLengths + 1], rest[kListLengths + 1], wave_total[kListThreads / kWave];
    const uint32_t t = threadIdx.x, lane = lane_id(), wave = wave_id();
    if (!check_bounds(bounds, sequences, tokens, status)) {  // (sequences that overlap could have more pieces than there is room for)
        for (uint32_t i = t; i < pieces; i += kListThreads) list[i] = make_uint4(0, 0, 0, 1);
        return;
    }
    uint32_t shift = 0;                                      // lengths are told apart to 2^shift pieces
    while ((tokens / kPieceRows + 1) >> shift >= kListLengths) ++shift;
    for (uint32_t i = t; i <= kListLengths; i += kListThreads) whole[i] = rest[i] = 0;
    __syncthreads();
    const auto sequence = [&](uint32_t s) {
        const uint32_t lo = umin(bounds[s], tokens);
        return make_uint2(lo, umax(lo, umin(bounds[s + 1], tokens)));
    };
    for (uint32_t s = t; s < sequences; s += kListThreads) {
        const uint2 q = sequence(s);
        const uint32_t n = (q.y - q.x + kPieceRows - 1) / kPieceRows;
        atomicAdd(&whole[n >> shift], 1u);                   // a sequence of n pieces has one of every length below n
        atomicAdd(&rest[n >> shift], n & ((1u << shift) - 1));
    }
    __syncthreads();
    // Pieces longer than length class k, for every k: class k holds 2^shift of every sequence that has a longer class, and the rest of those that end in it.
    const uint32_t k = kListLengths - 1 - t;                 // (threads go through the classes from the top)
    const uint32_t above = wave_scan_add(whole[k + 1]);      // sequences of the classes above k, within the wave
    if (lane == kWave - 1) wave_total[wave] = above;
    __syncthreads();
    uint32_t longer = above;
    for (uint32_t i = 0; i < wave; ++i) longer += wave_total[i];
    const uint32_t here = (longer << shift) + rest[k], upto = wave_scan_add(here);
    __syncthreads();
    if (lane == kWave - 1) wave_total[wave] = upto;
    __syncthreads();
    uint32_t at = upto - here;
    for (uint32_t i = 0; i < wave; ++i) at += wave_total[i];
    whole[k] = at;                                           // (every thread has read whole[k + 1] before the barriers above)
    __syncthreads();
    for (uint32_t s = wave; s < sequences; s += kListThreads / kWave) {
        const uint2 q = sequence(s);
        const uint32_t n = (q.y - q.x + kPieceRows - 1) / kPieceRows;
        for (uint32_t i = lane; i < n; i += kWave) {
            const uint32_t to = atomicAdd(&whole[i >> shift], 1u);
            if (to < pieces) list[to] = make_uint4(q.x, q.y, i, 0);
        }
    }
    __syncthreads();
    // Behind them the padding's pieces, then entries of nothing.
    const uint32_t end = umin(bounds[sequences], tokens), used = whole[0], padding = (tokens - end + kPieceRows - 1) / kPieceRows;
    for (uint32_t i = t; used + i < pieces; i += kListThreads) list[used + i] = i < padding ? make_uint4(end, tokens, i, 1) : make_uint4(0, 0, 0, 1);
}

void launch_attention_list(const uint32_t* bounds, uint32_t sequences, uint32_t tokens, uint32_t pieces, uint4* list, uint32_t* status, hipStream_t stream)
{
    hipLaunchKernelGGL(attention_list, dim3(1), dim3(kListThreads), 0, stream, bounds, sequences, tokens, pieces, list, status);
}

}  // namespace stalloc

using namespace stalloc;

namespace {

template <typename T> void launch_attention(const stalloc_attention_shape* s, const AttentionArgs<T>& a, uint32_t blocks, hipStream_t stream)
{
    const auto one = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kAttnThreads), 0, stream, a); };
    if (s->head_dim == 128) one(attention_rows<T, 128, true>);
    else if (s->head_dim > 64) one(attention_rows<T, 128, false>);
    else if (s->head_dim == 64) one(attention_rows<T, 64, true>);
    else one(attention_rows<T, 64, false>);
}

}  // namespace

extern "C" int stalloc_attention(const stalloc_attention_shape* shape, const stalloc_heads* q, const stalloc_heads* k,
                                 const stalloc_heads* v, const uint32_t* bounds, const stalloc_heads* o, float* lse,
                                 uint32_t* device_status, void* workspace, size_t* workspace_bytes, void* hip_stream)
{
    if (!shape_ok(shape) || !workspace_bytes) return STALLOC_ERR_INVALID_ARG;
    const uint32_t parts = parts_of(row_pieces(shape) * shape->heads, average_rows(shape) / kAttnKeys, kLeastSteps, 8);
    const uint64_t pieces = most_pieces(shape->tokens, shape->sequences, kAttnRows), blocks = pieces * shape->heads * parts;
    const uint64_t rows = (uint64_t)shape->tokens * shape->heads;
    if (blocks * kAttnThreads > kMostThreads) return STALLOC_ERR_TOO_LARGE;
    Carver cv(workspace);
    float* partial = cv.take<float>(parts > 1 ? parts * rows * shape->head_dim : 0);
    f32x2* part_stats = cv.take<f32x2>(parts > 1 ? parts * rows : 0);
    uint4* list = cv.take<uint4>(list_pays(blocks, shape->sequences) ? pieces : 1);
    if (!workspace) { *workspace_bytes = cv.used; return STALLOC_OK; }
    if (!heads_ok(q, shape, shape->heads, false) || !heads_ok(k, shape, shape->kv_heads, false) || !heads_ok(v, shape, shape->kv_heads, false) ||
        !heads_ok(o, shape, shape->heads, true) || !bounds || !lse || !device_status || *workspace_bytes < cv.used || !aligned(workspace, kAlign))
        return STALLOC_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    begin_launches();
    if (list_pays(blocks, shape->sequences)) launch_attention_list(bounds, shape->sequences, shape->tokens, (uint32_t)pieces, list, device_status, stream);
    else list = nullptr;
    with_type(shape->dtype, [&](auto t) {
        using T = decltype(t);
        if constexpr (sizeof(T) == 2) {
            const AttentionArgs<T> a = {heads_of<T>(q), heads_of<T>(k), heads_of<T>(v), heads_of<T>(o), lse, device_status,
                                        {list, bounds, shape->sequences, shape->tokens, (uint32_t)pieces, shape->heads, parts},
                                        partial, part_stats, shape->heads / shape->kv_heads, shape->head_dim, shape->scale};
            launch_attention<T>(shape, a, (uint32_t)blocks, stream);
            if (parts > 1) hipLaunchKernelGGL(attention_join<T>, dim3((uint32_t)((rows * (shape->head_dim / 8) + 255) / 256)), dim3(256), 0, stream, a);
        }
    });
    return launched();
}
