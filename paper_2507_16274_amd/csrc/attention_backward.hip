// stalloc_attention_backward: gradients of causal attention over packed sequences, weights computed again from lse.
//
//     p_ij = exp(scale q_i . k_j - lse_i),  D_i = do_i . o_i,  ds_ij = scale p_ij (do_i . v_j - D_i)
//     dq_i = sum_j ds_ij k_j,   dk_j = sum_h sum_i ds_ij q_i,   dv_j = sum_h sum_i p_ij do_i
//
// Two kernels: D and dq, a workgroup per 128 rows of a head; then dk and dv, a workgroup per 128 keys that goes through all rows that see them, of
// all heads that share them.  Scores are computed twice (seven products instead of five), and in return every sum belongs to one wave: no atomics, and the same
// result every time; partial gradients are in memory only where walks are cut into parts, because pieces and heads alone would not fill the chip.
//
// Bound like the forward kernel.  One sequence of 4096, 32 heads of 128: 0.20 ms and 0.30, matrix pipe busy 60 and 57 %; forward and backward pass 605 us, 0.80 PFLOP/s of the
// five products and the forward pass' two, 1.02 with what is made twice.
#include <type_traits>

#include "attention.h"

namespace stalloc {

template <typename T> struct AttentionBackwardArgs {
    Heads<T> d_o, q, k, v, o, dq, dk, dv;
    const float* lse;
    float* stats;                                            // [heads][2][tokens]: lse in units of log 2, -D (see kFarLse)
    uint32_t* status;
    Work rows, keys;                                         // shared out for dq; for dk and dv
    float* partial;                                          // [parts][2][kv_heads][tokens][head_dim]: dk, dv of a part, if there are several
    float* partial_dq;                                       // [parts][heads][tokens][head_dim]
    uint32_t tokens, heads, group, head_dim;
    float scale;
};

// Tiles of a part at least: of the walk over rows (which goes through several heads, so its parts are few tiles of each), of the walk over keys.
constexpr uint32_t kLeastRowSteps = 2, kLeastKeySteps = 4;
constexpr int kAbThreads = 256, kAbRows = kPieceRows, kAbStep = 32, kAbStages = 4;

// Rows near the beginning of a sequence see few keys: their weights and with them their ds are the largest of all, and dp - D is a difference of numbers as large
// as o.  There the rounding of o (in D) and of ds (as an operand) to 16 bits is what gradients lose, so the first kAbRows rows of a sequence, one
// piece of it, take D from sum_j p_ij dp_ij in 32 bits instead, by a walk of its own over at most four tiles, and multiply by ds in two parts: rounded, and what
// that left.  Relative to its norm dq of 600 rows of 64 in half precision is 0.00025 off, instead of 0.00033 (0.00021 if only the result were rounded).  It costs nothing that
// can be measured in one sequence of 4096, 2 % where 17 sequences share 5003 tokens, and 32 -> 38 us of both passes where 20 share 500.

// What rounding registers 8 s .. 8 s + 7 to T leaves of them.
template <typename T, int s> __device__ __forceinline__ V8<T> left_of(const f32x16& x, V8<T> rounded)
{
    const f32x8 v = {x[8 * s], x[8 * s + 1], x[8 * s + 2], x[8 * s + 3], x[8 * s + 4], x[8 * s + 5], x[8 * s + 6], x[8 * s + 7]};
    return __builtin_convertvector(v - __builtin_convertvector(rounded, f32x8), V8<T>);
}

// What the loops leave out: dp - D is made by the products, whose sum begins at -D, and scale is multiplied in when results are stored (that and the sums' own beginning are
// 32 of 160 vector operations a step; one sequence of 4096 with 32 heads of 128: 623 us both passes with them, 603 without).

// Where lse is large, 32 bits of it say too little: beyond 2^16 (in units of log 2) its rounding is half a per cent of every weight, from 2^24 on whole powers of two.  Rows like that have
// their maximum and sum made again, pair by pair, and so are all their weights: their lse in `stats` is a NaN, which sends what they reach to rows_again and keys_again, with log2
// of the sum as its payload, and in place of -D is the maximum.  So are rows whose scores are all -infinity and that have no weights: NaN throughout.
constexpr float kFarLse = 1 << 16;

struct RowWeights {
    float lse2, m, log_total;                                // lse2 is NaN: by the maximum and the sum
    __device__ __forceinline__ float operator()(float s, float scale, float lift = 0.f) const
    {
        return exp2_fast(lse2 != lse2 ? (s - m) * scale - log_total : __builtin_fmaf(s, scale, -lse2) - lift);
    }
};
__device__ __forceinline__ float packed(float log_total) { return as_float(0x7fc00000u | ((as_bits(log_total) + 256) >> 9 & 0x3fffffu)); }
__device__ __forceinline__ float unpacked(float lse2) { return as_float((as_bits(lse2) & 0x3fffffu) << 9); }

// Half precision: numbers that are multiplied again have to lie among the type's normal ones, 2^-14 to 2^16.  Weights, at most 1 and as small as 1 / row, are lifted by 2^14: lse in
// `stats` is less by 14, and dv is divided by as much at last.  Their gradients ds have the size of d_o, whatever that is.  They are multiplied by a power of two, of each row in dq and
// of each key in dk, that is lowered when the next tile's largest would pass 2^14 (to where it is below 2^8), and the sums with it; the results are divided by it.  It begins at 2^60, for which
// nothing is too small.  Without it d_o of 10^-5, of the ordinary size of a mean loss' gradients, cost dq and dk 0.062 of their norm (rounding them 0.022), and d_o of 10^4 was beyond
// the type, though the results are not.  bfloat16 has the range of 32 bits.  It costs both passes 2 % (one sequence of 4096, 32 heads of 128: 628 -> 641 us) to 5 % (17 sequences, 5003 tokens, heads
// of 64: 131 -> 139); looking at the rounded operands instead, packed, saves instructions and no time.
template <typename T> constexpr bool kNarrow = std::is_same<T, f16>::value;
template <typename T> constexpr float kLift = kNarrow<T> ? 14.f : 0.f;
constexpr float kMostDs = 16384.f, kMostFactor = 1152921504606846976.f;                   // 2^14, 2^60

__device__ __forceinline__ float largest(const f32x16& x)
{
    float t[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) t[i] = max3(fabsf(x[3 * i]), fabsf(x[3 * i + 1]), fabsf(x[3 * i + 2]));
    return fmaxf(max3(t[0], t[1], t[2]), max3(t[3], t[4], fabsf(x[15])));
}
// The exponent of the power of two that leaves 2^7 to 2^8 of t (finite; of an infinity nothing is left but NaN, which is made again).
__device__ __forceinline__ int exponent_for(float t) { return __builtin_amdgcn_frexp_expf(t) - 8; }

// dk and dv of a wave's keys pair by pair (attention.h): `steps` steps of the walk from `from_step` on.
template <typename T, int kD, bool kFull>
__device__ __forceinline__ void keys_again(const AttentionBackwardArgs<T>& a, const Piece& p, uint32_t kv, uint32_t from_step, uint32_t steps, f32x16 (&dk)[kD / 32],
                                           f32x16 (&dv)[kD / 32])
{
    const uint32_t first = p.first + 32 * wave_id(), key = first + (lane_id() & 31), last = p.end - 1, per_head = (p.end - p.first + kAbStep - 1) / kAbStep;
    V8<T> k[kD / 16], v[kD / 16];
    load_row<T, kD, kFull>(k, a.k.at(umin(key, last), kv), a.head_dim);
    load_row<T, kD, kFull>(v, a.v.at(umin(key, last), kv), a.head_dim);
#pragma unroll
    for (int d = 0; d < kD / 32; ++d) dk[d] = dv[d] = f32x16{};
    for (uint32_t step = from_step; step < from_step + steps; ++step) {
        const uint32_t head = kv * a.group + step / per_head, begin = p.first + step % per_head * kAbStep;
#pragma unroll 1
        for (uint32_t row = umax(begin, first); row < umin(begin + kAbStep, p.end); ++row) {
            const T* q = a.q.at(row, head);
            const T* d_o = a.d_o.at(row, head);
            const float s = dot_row<T, kD, kFull>(k, q, a.head_dim), dp = dot_row<T, kD, kFull>(v, d_o, a.head_dim);
            const float* stats = a.stats + (uint64_t)head * 2 * a.tokens + row;
            const RowWeights weights = {stats[0], stats[a.tokens], unpacked(stats[0])};
            float less_d = stats[a.tokens];
            if (weights.lse2 != weights.lse2) {
                float d = 0.f;
#pragma unroll 1
                for (uint32_t col = lane_id(); col < a.head_dim; col += kWave) d = __builtin_fmaf((float)a.o.at(row, head)[col], (float)d_o[col], d);
                less_d = -wave_sum(d);
            }
            const float w = weights(s, a.scale * kLog2e, kLift<T>);
            if (row < key) continue;
            add_row<T, kD, kFull>(dv, w, d_o, a.head_dim);
            add_row<T, kD, kFull>(dk, w * (dp + less_d), q, a.head_dim);
        }
        if (__all(key >= p.end || (all_nan(dk, a.head_dim) && all_nan(dv, a.head_dim)))) return;
    }
}

template <typename T, int kD, bool kFull> __global__ void __launch_bounds__(kAbThreads, kD == 64 ? 3 : 2) attention_dk_dv(AttentionBackwardArgs<T> a)
{
    __shared__ __attribute__((aligned(256))) T ring[kAbStages][2][kAbStep * kD];           // rows of q, of d_o
    __shared__ __attribute__((aligned(16))) float ring_stats[kAbStages][kAbThreads / kWave][2][kAbStep];     // (a copy per wave)
    if (blockIdx.x == 0 && !a.keys.list) check_bounds(a.keys.bounds, a.keys.sequences, a.tokens, a.status);
    const Task task = take_task<kAbRows, false>(a.keys);
    const Piece p = task.piece;
    const uint32_t kv = task.head, parts = a.keys.parts;
    if (p.first >= p.end) return;
    const uint32_t half = lane_id() >> 5, first = p.first + 32 * wave_id(), key = first + (lane_id() & 31);
    f32x16 dk[kD / 32] = {}, dv[kD / 32] = {};
    float factor = kNarrow<T> ? kMostFactor : 1.f;           // of ds, that is in dk
    float lift = kNarrow<T> ? 16384.f : 1.f;                 // of weights, that is in dk and dv
    if (!p.no_keys) {
        const uint32_t last = p.end - 1;
        const float scale = uniform(a.scale * kLog2e);
        using Tile = Rows<T, kD, kAbStep, kAbThreads, kFull>;
        constexpr uint32_t kTile = sizeof(ring[0][0]);
        const Places<kD> places;
        // The walk: the rows from p.first on, of one head after the other; this part's share of it.
        const uint32_t per_head = (p.end - p.first + kAbStep - 1) / kAbStep, all = per_head * a.group;
        const uint32_t from_step = (uint32_t)((uint64_t)all * task.part / parts), steps = (uint32_t)((uint64_t)all * (task.part + 1) / parts) - from_step;
        uint32_t next_head = kv * a.group + from_step / per_head, next_row = p.first + from_step % per_head * kAbStep, next_slot = 0;
        const float* lane_stats = a.stats + (uint64_t)half * a.tokens + (lane_id() & 31);
        const auto fetch = [&]() {
            Tile::fetch(ring[next_slot][0], a.q.at(0, next_head), a.q.token, next_row, last, a.head_dim);
            Tile::fetch(ring[next_slot][1], a.d_o.at(0, next_head), a.d_o.token, next_row, last, a.head_dim);
            words_to_lds(lds_address(ring_stats[next_slot][wave_id()]), lane_stats + (uint64_t)next_head * 2 * a.tokens + next_row);
            next_row += kAbStep;
            if (next_row >= p.end) { next_row = p.first; ++next_head; }
            next_slot = (next_slot + 1) % kAbStages;
        };
        constexpr int kLoads = 2 * Tile::kLoads + 1;
        if (!kFull) clear_lds<sizeof(ring) / 4, kAbThreads>(ring);
        uint32_t row = next_row, now = 0;
        for (uint32_t step = 0; step < kAbStages - 1 && step < steps; ++step) fetch();
        V8<T> k[kD / 16], v[kD / 16];
        load_row<T, kD, kFull>(k, a.k.at(umin(key, last), kv), a.head_dim);
        load_row<T, kD, kFull>(v, a.v.at(umin(key, last), kv), a.head_dim);
        vector_memory_done();                                // (these are here before the loop: their loads are not waited for among the tiles')
        // Two loops, that pieces without early rows do not pay for them: one sequence of 4096 with 32 heads of 128 took 644 us both passes with one loop, 629 with two.
        const auto walk = [&](auto early) {
            for (uint32_t step = 0; step < steps; ++step) {
                if (step + kAbStages - 1 < steps) {
                    tiles_landed<kLoads * (kAbStages - 2)>();
                    fetch();
                } else {
                    tiles_landed<0>();
                }
                const uint32_t along = kept(now * 2 * kTile + places.along), cross = kept(now * 2 * kTile + places.cross);
                const float (*stats)[kAbStep] = ring_stats[now][wave_id()];
                if (row + kAbStep - 1 >= first && first < p.end) {       // (else none of these rows sees a key of this wave, or it has no keys)
                    f32x16 s = {}, dp;
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
#pragma unroll
                        for (int j = 0; j < 4; ++j) dp[i + j] = (*(const Vec<float>::x4*)&stats[1][row_of(i, half)])[j];
                    products<kD / 8, 3, T, 1>([&](int i) { return read_along<T, kD>(ring[0][0], along, i / 2, i % 2 * kTile); },
                                           [&](int i, V8<T> r) {
                                               if (i % 2 == 0) s = mma(r, k[i / 2], s);
                                               else dp = mma(r, v[i / 2], dp);
                                           });
                    const bool crosses = row < first + 31 || row + kAbStep > p.end;      // some of these rows do not see some of these keys, or are not the sequence's
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const Vec<float>::x4 lse2 = *(const Vec<float>::x4*)&stats[0][row_of(i, half)];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            s[i + j] = exp2_fast(__builtin_fmaf(s[i + j], scale, -lse2[j]));
                            dp[i + j] *= s[i + j];
                        }
                    }
                    if (crosses)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t r = row + row_of(i, half);
                            if (r < key || r >= p.end) s[i] = dp[i] = 0.f;
                        }
                    if constexpr (kNarrow<T>) {
                        dp *= factor;
                        const float t = largest(dp);
                        if (__any(t > kMostDs)) {
                            const float most = fmaxf(t, across(t)), f = __builtin_amdgcn_ldexpf(1.f, most > kMostDs ? -exponent_for(most) : 0);
                            factor *= f;
                            dp *= f;
#pragma unroll
                            for (int d = 0; d < kD / 32; ++d) dk[d] *= f;
                        }
                    }
                    // Weights and their gradients are rounded to T for the products; sums stay in 32 bits.
                    const V8<T> w[2] = {operand<T, 0>(s), operand<T, 1>(s)}, ds[2] = {operand<T, 0>(dp), operand<T, 1>(dp)};
                    if (early && row < p.begin + kAbRows) {
                        const V8<T> left[2] = {left_of<T, 0>(dp, ds[0]), left_of<T, 1>(dp, ds[1])};
                        products<kD / 16, 2, T, 1>([&](int i) { return read_cross<T, kD>(ring[0][0], cross, i / 2, i % 2 * 32 * kD); },
                                                [&](int i, V8<T> r) { dk[i / 2] = mma(r, left[i % 2], dk[i / 2]); });
                    }
                    products<kD / 8, 4, T, 1>([&](int i) { return read_cross<T, kD>(ring[0][0], cross, i / 4, i % 2 * kTile + i / 2 % 2 * 32 * kD); },
                                           [&](int i, V8<T> r) {
                                               if (i % 2 == 0) dk[i / 4] = mma(r, ds[i / 2 % 2], dk[i / 4]);
                                               else dv[i / 4] = mma(r, w[i / 2 % 2], dv[i / 4]);
                                           });
                }
                row += kAbStep;
                if (row >= p.end) row = p.first;
                now = (now + 1) % kAbStages;
            }
        };
        if (p.first == p.begin) walk(std::true_type{});
        else walk(std::false_type{});
        if (__any(not_finite(dk) || not_finite(dv))) {
            keys_again<T, kD, kFull>(a, p, kv, from_step, steps, dk, dv);
            factor = lift = 1.f;
        }
    }
    if (key >= p.end) return;
    const float unlift = 1.f / lift, unfactor = unlift / factor;
    if (parts > 1) {
        const uint64_t heads = a.keys.heads, to = ((2 * task.part * heads + kv) * a.tokens + key) * a.head_dim;
        store_row<float, kD, kFull>(a.partial + to, dk, a.scale * unfactor, a.head_dim);
        store_row<float, kD, kFull>(a.partial + to + heads * a.tokens * a.head_dim, dv, unlift, a.head_dim);
        return;
    }
    store_row<T, kD, kFull>(a.dk.at(key, kv), dk, a.scale * unfactor, a.head_dim);
    store_row<T, kD, kFull>(a.dv.at(key, kv), dv, unlift, a.head_dim);
}

// Tensors of `heads` heads from those of the parts, added up in their order: eight numbers a thread.  kTwo: two tensors, one behind the other in
// every part (dk, dv).
template <typename T, bool kTwo> __global__ void __launch_bounds__(256) gradient_join(const float* partial, uint32_t parts, uint32_t heads, uint32_t tokens, uint32_t head_dim, Heads<T> x, Heads<T> y)
{
    const uint64_t each = (uint64_t)heads * tokens * head_dim, all = kTwo ? 2 * each : each, at = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= all) return;
    f32x8 sum = load8(partial + at);
    for (uint32_t part = 1; part < parts; ++part) sum += load8(partial + part * all + at);
    const uint64_t in = at < each ? at : at - each, row = in / head_dim;
    const Heads<T>& to = at < each ? x : y;
    store8(to.at(row % tokens, (uint32_t)(row / tokens)) + in % head_dim, sum);
}

// dq of a wave's rows over keys from .. to - 1, pair by pair (attention.h).
template <typename T, int kD, bool kFull>
__device__ __forceinline__ void rows_again(const AttentionBackwardArgs<T>& a, const Piece& p, uint32_t head, uint32_t from, uint32_t to, RowWeights weights, float d, f32x16 (&dq)[kD / 32])
{
    const uint32_t first = p.first + 32 * wave_id(), row = first + (lane_id() & 31), last = p.end - 1, kv = head / a.group;
    V8<T> q[kD / 16], d_o[kD / 16];
    load_row<T, kD, kFull>(q, a.q.at(umin(row, last), head), a.head_dim);
    load_row<T, kD, kFull>(d_o, a.d_o.at(umin(row, last), head), a.head_dim);
#pragma unroll
    for (int d = 0; d < kD / 32; ++d) dq[d] = f32x16{};
#pragma unroll 1
    for (uint32_t key = from; key < umin(to, umin(first + 31, last) + 1); ++key) {
        const T* k = a.k.at(key, kv);
        const float s = dot_row<T, kD, kFull>(q, k, a.head_dim), dp = dot_row<T, kD, kFull>(d_o, a.v.at(key, kv), a.head_dim);
        const float w = weights(s, a.scale * kLog2e);
        if (key <= row) add_row<T, kD, kFull>(dq, w * (dp - d), k, a.head_dim);
        if (key % 32 == 0 && __all(all_nan(dq, a.head_dim))) return;
    }
}

// D of a wave's rows (one per lane, in q and d_o as load_row gives them), which are among the first kAbRows of a sequence: the keys' and values' tiles come
// straight from memory.
template <typename T, int kD, bool kFull>
__device__ __forceinline__ float early_d(const AttentionBackwardArgs<T>& a, const Piece& p, uint32_t kv, const V8<T> (&q)[kD / 16], const V8<T> (&d_o)[kD / 16], float lse2)
{
    const uint32_t half = lane_id() >> 5, first = p.first + 32 * wave_id(), row = first + (lane_id() & 31), last = p.end - 1;
    const float scale = uniform(a.scale * kLog2e);
    float sum = 0.f;
#pragma unroll 1
    for (uint32_t key = p.begin; key <= umin(first, last); key += 32) {
        const uint32_t mine = umin(key + (lane_id() & 31), last);
        V8<T> x[kD / 16], y[kD / 16];
        load_row<T, kD, kFull>(x, a.k.at(mine, kv), a.head_dim);
        load_row<T, kD, kFull>(y, a.v.at(mine, kv), a.head_dim);
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int c = 0; c < kD / 16; ++c) {
            s = mma(x[c], q[c], s);
            dp = mma(y[c], d_o[c], dp);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float w = exp2_fast(__builtin_fmaf(s[i], scale, -lse2));
            if (key + row_of(i, half) <= row) sum = __builtin_fmaf(w, dp[i], sum);
        }
    }
    return sum + across(sum);
}

template <typename T, int kD, bool kFull> __global__ void __launch_bounds__(kAbThreads, kD == 64 ? 3 : 2) attention_dq(AttentionBackwardArgs<T> a)
{
    __shared__ __attribute__((aligned(256))) T ring[kAbStages][2][kAbStep * kD];           // keys, values
    const Task task = take_task<kAbRows, true>(a.rows);
    const Piece p = task.piece;
    const uint32_t head = task.head;
    if (p.first >= p.end) return;
    const uint32_t half = lane_id() >> 5, first = p.first + 32 * wave_id(), row = first + (lane_id() & 31);
    f32x16 dq[kD / 32] = {};
    float factor = kNarrow<T> ? kMostFactor : 1.f;           // of ds, that is in dq
    if (!p.no_keys) {
        const uint32_t last = p.end - 1, kv = head / a.group, mine = umin(row, last);
        const T* k = a.k.at(0, kv);
        const T* v = a.v.at(0, kv);
        const float scale = uniform(a.scale * kLog2e);
        using Tile = Rows<T, kD, kAbStep, kAbThreads, kFull>;
        constexpr uint32_t kTile = sizeof(ring[0][0]);
        const Places<kD> places;
        // The walk: tiles of keys up to the last row's; this part's share of them.
        const uint32_t all = (umin(p.first + kAbRows, p.end) - p.begin + kAbStep - 1) / kAbStep;
        const uint32_t from = p.begin + (uint32_t)((uint64_t)all * task.part / a.rows.parts) * kAbStep;
        const uint32_t steps = (uint32_t)((uint64_t)all * (task.part + 1) / a.rows.parts) - (from - p.begin) / kAbStep;
        const auto fetch = [&](uint32_t step) {
            T (&stage)[2][kAbStep * kD] = ring[step % kAbStages];
            Tile::fetch(stage[0], k, a.k.token, from + step * kAbStep, last, a.head_dim);
            Tile::fetch(stage[1], v, a.v.token, from + step * kAbStep, last, a.head_dim);
        };
        if (!kFull) clear_lds<sizeof(ring) / 4, kAbThreads>(ring);
        for (uint32_t step = 0; step < kAbStages - 1 && step < steps; ++step) fetch(step);
        V8<T> q[kD / 16], d_o[kD / 16];
        load_row<T, kD, kFull>(q, a.q.at(mine, head), a.head_dim);
        load_row<T, kD, kFull>(d_o, a.d_o.at(mine, head), a.head_dim);
        // D_i of the lane's row, half of the columns each; for the kernel behind this one as well.
        V8<T> o[kD / 16];
        load_row<T, kD, kFull>(o, a.o.at(mine, head), a.head_dim);
        f32x2 stats = {a.lse[(uint64_t)head * a.tokens + mine] * kLog2e, 0.f};
#pragma unroll
        for (int c = 0; c < kD / 16; ++c) stats[1] += dot(__builtin_convertvector(o[c], f32x8), __builtin_convertvector(d_o[c], f32x8));
        stats[1] += across(stats[1]);
        const bool early = p.first == p.begin, far = !(fabsf(stats[0]) <= kFarLse);
        RowWeights weights = {stats[0], stats[0], 0.f};
        if (__any(far && stats[0] == stats[0])) {
            const f32x2 again = row_stats<T, kD, kFull>(q, k, a.k.token, p.begin, umin(first + 31, last) + 1, mine, scale, a.head_dim);
            if (far && stats[0] == stats[0]) weights = {packed(log2f(again[1])), again[1] > 0.f ? again[0] : as_float(0x7fc00000u), log2f(again[1])};
            stats[0] = weights.lse2;
        }
        if (early) {
            const float d = early_d<T, kD, kFull>(a, p, kv, q, d_o, stats[0]);
            if (!far) stats[1] = d;
        }
        if (row < p.end && task.part == 0) a.stats[((uint64_t)head * 2 + half) * a.tokens + row] = half == 0 ? (far ? stats[0] : stats[0] - kLift<T>) : far ? weights.m : -stats[1];
        float less = kNarrow<T> ? stats[0] - 60.f : stats[0];        // lse2, and the logarithm of the divisor
        f32x16 less_d = f32x16{} - stats[1];
        asm volatile("" : "+v"(less_d));                     // (in registers, not made anew every step)
        vector_memory_done();
        for (uint32_t step = 0; step < steps; ++step) {
            const uint32_t key = from + step * kAbStep;
            if (step + kAbStages - 1 < steps) {
                tiles_landed<2 * Tile::kLoads * (kAbStages - 2)>();
                fetch(step + kAbStages - 1);
            } else {
                tiles_landed<0>();
            }
            const uint32_t tile = step % kAbStages * 2 * kTile, along = kept(tile + places.along), cross = kept(tile + places.cross);
            if (key > first + 31 || first >= p.end) continue;        // (none of the wave's rows sees any of these keys, or it has no rows)
            f32x16 s = {}, dp = less_d;
            products<kD / 8, 4, T, 1>([&](int i) { return read_along<T, kD>(ring[0][0], along, i / 2, i % 2 * kTile); },
                                   [&](int i, V8<T> r) {
                                       if (i % 2 == 0) s = mma(r, q[i / 2], s);
                                       else dp = mma(r, d_o[i / 2], dp);
                                   });
            const bool crosses = key + 31 > first;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                dp[i] *= exp2_fast(__builtin_fmaf(s[i], scale, -less));
            }
            if (crosses)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key + row_of(i, half) > row) dp[i] = 0.f;
            if constexpr (kNarrow<T>) {
                const float t = largest(dp);
                if (__any(t > kMostDs)) {
                    const float most = fmaxf(t, across(t));
                    const int by = most > kMostDs ? exponent_for(most) : 0;
                    const float f = __builtin_amdgcn_ldexpf(1.f, -by);
                    factor *= f;
                    less += (float)by;
                    dp *= f;
#pragma unroll
                    for (int d = 0; d < kD / 32; ++d) dq[d] *= f;
                }
            }
            const V8<T> ds[2] = {operand<T, 0>(dp), operand<T, 1>(dp)};
            constexpr int kDs = kD / 32;
            if (early) {
                const V8<T> left[2] = {left_of<T, 0>(dp, ds[0]), left_of<T, 1>(dp, ds[1])};
                products<2 * kDs, 2, T, 1>([&](int i) { return read_cross<T, kD>(ring[0][0], cross, i % kDs, i / kDs * 32 * kD); },
                                        [&](int i, V8<T> r) { dq[i % kDs] = mma(r, left[i / kDs], dq[i % kDs]); });
            }
            products<2 * kDs, 4, T, 1>([&](int i) { return read_cross<T, kD>(ring[0][0], cross, i % kDs, i / kDs * 32 * kD); },
                                    [&](int i, V8<T> r) { dq[i % kDs] = mma(r, ds[i / kDs], dq[i % kDs]); });
        }
        if (__any(not_finite(dq))) {
            rows_again<T, kD, kFull>(a, p, head, from, from + steps * kAbStep, weights, stats[1], dq);
            factor = 1.f;
        }
    }
    if (row >= p.end) return;
    if (a.rows.parts > 1) store_row<float, kD, kFull>(a.partial_dq + (((uint64_t)task.part * a.heads + head) * a.tokens + row) * a.head_dim, dq, a.scale / factor, a.head_dim);
    else store_row<T, kD, kFull>(a.dq.at(row, head), dq, a.scale / factor, a.head_dim);
}

}  // namespace stalloc

using namespace stalloc;

namespace {

template <typename T, int kD, bool kFull> void launch_backward(const AttentionBackwardArgs<T>& a, hipStream_t stream)
{
    hipLaunchKernelGGL((attention_dq<T, kD, kFull>), dim3(a.rows.pieces * a.heads * a.rows.parts), dim3(kAbThreads), 0, stream, a);
    hipLaunchKernelGGL((attention_dk_dv<T, kD, kFull>), dim3(a.keys.pieces * a.keys.heads * a.keys.parts), dim3(kAbThreads), 0, stream, a);
}

template <typename T> void launch_joins(const AttentionBackwardArgs<T>& a, hipStream_t stream)
{
    const auto blocks = [&](uint32_t heads) { return dim3((uint32_t)(((uint64_t)heads * a.tokens * a.head_dim / 8 + 255) / 256)); };
    if (a.rows.parts > 1)
        hipLaunchKernelGGL((gradient_join<T, false>), blocks(a.heads), dim3(256), 0, stream, a.partial_dq, a.rows.parts, a.heads, a.tokens, a.head_dim, a.dq, a.dq);
    if (a.keys.parts > 1)
        hipLaunchKernelGGL((gradient_join<T, true>), blocks(2 * a.keys.heads), dim3(256), 0, stream, a.partial, a.keys.parts, a.keys.heads, a.tokens, a.head_dim, a.dk, a.dv);
}

}  // namespace

extern "C" int stalloc_attention_backward(const stalloc_attention_shape* shape, const stalloc_heads* d_o, const stalloc_heads* q,
                                          const stalloc_heads* k, const stalloc_heads* v, const stalloc_heads* o, const float* lse,
                                          const uint32_t* bounds, const stalloc_heads* dq, const stalloc_heads* dk,
                                          const stalloc_heads* dv, uint32_t* device_status, void* workspace,
                                          size_t* workspace_bytes, void* hip_stream)
{
    if (!shape_ok(shape) || !workspace_bytes) return STALLOC_ERR_INVALID_ARG;
    const uint32_t heads = shape->heads, kv = shape->kv_heads;
    const uint32_t parts = parts_of(row_pieces(shape) * kv, average_rows(shape) / kAbStep * (heads / kv), kLeastRowSteps, 16);
    const uint32_t row_parts = parts_of(row_pieces(shape) * heads, average_rows(shape) / kAbStep, kLeastKeySteps, 8);
    const uint64_t pieces = most_pieces(shape->tokens, shape->sequences, kAbRows);
    const uint64_t joined = 2 * (uint64_t)kv * shape->tokens * shape->head_dim;
    if (pieces * heads * row_parts * kAbThreads > kMostThreads || pieces * kv * parts * kAbThreads > kMostThreads) return STALLOC_ERR_TOO_LARGE;
    const bool listed = list_pays(pieces * heads, shape->sequences);
    Carver cv(workspace);
    float* stats = cv.take<float>(2 * (size_t)shape->tokens * heads + kAbStep);
    uint4* list = cv.take<uint4>(listed ? pieces : 0);
    float* partial = cv.take<float>(parts > 1 ? parts * joined : 0);
    float* partial_dq = cv.take<float>(row_parts > 1 ? (uint64_t)row_parts * heads * shape->tokens * shape->head_dim : 0);
    if (!workspace) { *workspace_bytes = cv.used; return STALLOC_OK; }
    if (!heads_ok(d_o, shape, heads, false) || !heads_ok(q, shape, heads, false) || !heads_ok(k, shape, kv, false) || !heads_ok(v, shape, kv, false) ||
        !heads_ok(o, shape, heads, false) || !heads_ok(dq, shape, heads, true) || !heads_ok(dk, shape, kv, true) || !heads_ok(dv, shape, kv, true) ||
        !lse || !bounds || !device_status || *workspace_bytes < cv.used || !aligned(workspace, kAlign))
        return STALLOC_ERR_INVALID_ARG;
    if (dq->data == q->data || dq->data == d_o->data || dq->data == o->data) return STALLOC_ERR_INVALID_ARG;       // (they are read again when dq is written)
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    begin_launches();
    if (listed) launch_attention_list(bounds, shape->sequences, shape->tokens, (uint32_t)pieces, list, device_status, stream);
    else list = nullptr;
    const Work by_rows = {list, bounds, shape->sequences, shape->tokens, (uint32_t)pieces, heads, row_parts};
    const Work by_keys = {list, bounds, shape->sequences, shape->tokens, (uint32_t)pieces, kv, parts};
    with_type(shape->dtype, [&](auto t) {
        using T = decltype(t);
        if constexpr (sizeof(T) == 2) {
            const AttentionBackwardArgs<T> a = {heads_of<T>(d_o), heads_of<T>(q), heads_of<T>(k), heads_of<T>(v), heads_of<T>(o), heads_of<T>(dq),
                                                heads_of<T>(dk), heads_of<T>(dv), lse, stats, device_status, by_rows, by_keys, partial, partial_dq, shape->tokens,
                                                heads, heads / kv, shape->head_dim, shape->scale};
            if (shape->head_dim == 128) launch_backward<T, 128, true>(a, stream);
            else if (shape->head_dim > 64) launch_backward<T, 128, false>(a, stream);
            else if (shape->head_dim == 64) launch_backward<T, 64, true>(a, stream);
            else launch_backward<T, 64, false>(a, stream);
            launch_joins<T>(a, stream);
        }
    });
    return launched();
}
