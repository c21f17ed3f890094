// What the attention kernels share: matrix products of 32 x 32 tiles, tiles in LDS, and which rows of which sequence a workgroup takes.
//
// v_mfma_f32_32x32x16 multiplies A (32 rows x 16) by B (16 x 32 columns).  Lane l holds of A the row l % 32 and of B the
// column l % 32, both at the positions 8 (l / 32) .. + 7 of the 16; of the result it holds the column l % 32 and the rows
// 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15.  A result with keys as rows is therefore, registers 0 .. 7 and 8 .. 15
// taken as they are, the B operand of a product over these keys, if the other operand takes the keys in the same order:
// positions 0 .. 3 and 4 .. 7 of half h = l / 32 stand for keys 4 h + 0 .. 3 and 8 + 4 h + 0 .. 3.  So weights never leave the
// registers of the lane that made them.
#pragma once

#include "numbers.h"

namespace stalloc {

template <typename T> using V4 = typename Vec<T>::x4;
template <typename T> using V8 = typename Vec<T>::x8;

__device__ __forceinline__ f32x16 mma(V8<bf16> a, V8<bf16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(V8<f16> a, V8<f16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int kOthersMayMove = 0x2 | 0x4;                    // vector and scalar instructions, not memory accesses and matrix products

// Registers 8 s .. 8 s + 7 of a result, rounded to T, as the operand of the next product.
template <typename T, int s> __device__ __forceinline__ V8<T> operand(const f32x16& x)
{
    const f32x8 v = {x[8 * s], x[8 * s + 1], x[8 * s + 2], x[8 * s + 3], x[8 * s + 4], x[8 * s + 5], x[8 * s + 6], x[8 * s + 7]};
    return __builtin_convertvector(v, V8<T>);
}

// The row (of the result tile) that register i of a lane holds.
__device__ __forceinline__ uint32_t row_of(int i, uint32_t half) { return 8 * (i / 4) + 4 * half + i % 4; }

// The same lane of the other half of the wave.
__device__ __forceinline__ float across(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
    return as_float(lane_id() < 32 ? r[1] : r[0]);
}

// A tile of rows of kD numbers in LDS.  16-byte pieces of a row change places with the row's number, so that lanes in different rows at one column
// reach different banks (64 of 4 bytes, a row of 128 numbers takes all of them) both in reads along a row, 16 rows at
// a time, and in transposing reads, 64 bytes of each of four neighbouring rows at a time: the low bits of the row move blocks of
// four pieces, the next ones pieces within a block.  (Moving pairs of pieces by the row's low bits cost two further cycles a
// transposing read and four a read along a row: one sequence of 8192 with 64 heads went from 1119 to 1091 us without them.)
template <int kD> __device__ __forceinline__ uint32_t turn_of(uint32_t row)
{
    return kD == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// Where a lane reads in a tile, in bytes.  The columns that a read is for only change bits that the tile's place does not reach: they are put in
// by an exclusive or where the read is, which costs an instruction and saves the registers of all the places.
//   along  its row l % 32, numbers 8 (l / 32) .. + 7; columns 16 c further on: along ^ 32 c
//   cross  of a transposing read, in which lane i of 16 gets the i-th column of four rows whose quarters its neighbours point at: column l % 32, rows
//          4 (l / 32) .. + 3; columns 32 d further on: cross ^ 64 d; eight rows further on: (cross ^ 32) + 16 kD
template <int kD> struct Places {
    uint32_t along, cross;
    __device__ __forceinline__ Places()
    {
        const uint32_t l = lane_id(), row = l & 31, half = l >> 5, i = l & 15, from = 4 * half + (i >> 2), col = 16 * ((l >> 4) & 1) + 4 * (i & 3);
        along = row * kD * 2 + ((half ^ turn_of<kD>(row)) << 4);
        cross = from * kD * 2 + (((col >> 3) ^ turn_of<kD>(from)) << 4) + (col & 7) * 2;
    }
};

// A number that is the same in all lanes, in a scalar register.
__device__ __forceinline__ float uniform(float v) { return as_float(__builtin_amdgcn_readfirstlane(as_bits(v))); }

// A sum as it is, in a register: merged with the exclusive ors behind it, each of their constants would take a register of its own.
__device__ __forceinline__ uint32_t kept(uint32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// The A operand of a product over columns 16 c .. + 15 of the rows l % 32 of the tile that lies `tile` bytes behind `ring`.
template <typename T, int kD> __device__ __forceinline__ V8<T> read_along(const T* ring, uint32_t along_in_tile, int c, uint32_t further = 0)
{
    return *(const V8<T>*)((const char*)ring + ((along_in_tile ^ (32 * c)) + further));
}

// The A operand of a product over 16 rows (`further`: bytes to the first of them, whole multiples of 16 rows) for columns 32 d .. + 31: lane l gets
// column 32 d + l % 32 and the rows in the order of `operand`.
template <typename T, int kD> __device__ __forceinline__ V8<T> read_cross(const T* ring, uint32_t cross_in_tile, int d, uint32_t further = 0)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const uint32_t at = cross_in_tile ^ (64 * d);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)((const char*)ring + (at + further)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)((const char*)ring + ((at ^ 32) + further + 16 * kD)));
    const V4<T> a = __builtin_bit_cast(V4<T>, lo), b = __builtin_bit_cast(V4<T>, hi);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// 16 bytes per lane from memory to LDS, lane after lane from `lds` on; `base` and `lds` are the same in all lanes.  Written out because
// the compiler, which cannot know that the tile asked for is not the one read next, would wait for it there and then; what waits
// for it is tiles_landed.  Nothing is returned in registers.  A memory access may read a scalar register five wait states after a vector instruction (a readfirstlane) has written it
// and not before; the compiler, which sees to that elsewhere, does not look into assembly, so the five are in it.  The place in LDS is in m0,
// where the compiler puts it, so that it knows.
__device__ __forceinline__ void memory_to_lds(uint32_t lds, const void* base, uint32_t offset)
{
    const uint64_t from = uniform((uint64_t)base);
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(from), "{m0}"(lds) : "memory");
}
// The same, 4 bytes from an address of each lane's own.
__device__ __forceinline__ void words_to_lds(uint32_t lds, const void* from)
{
    asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, off" ::"v"(from), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return uniform((uint32_t)(size_t)(__attribute__((address_space(3))) const void*)p); }

// kRows rows of a tensor on their way to LDS, without a register between: the memory pipe writes 64 lanes' pieces one behind the other, so a lane asks
// for the piece that belongs where its own lands.  Rows past `last` repeat it; columns from head_dim on are left as they are (the
// kernel has cleared them).  `first` <= `last`; kLoads accesses of every wave, counted by vmcnt.
template <typename T, int kD, int kRows, int kThreads, bool kFull> struct Rows {
    static constexpr int kPieces = kD / 8, kLoads = kRows * kPieces / kThreads;
    static_assert(kLoads * kThreads == kRows * kPieces, "whole accesses");

    static __device__ __forceinline__ void fetch(T* tile, const T* data, uint64_t stride, uint32_t first, uint32_t last, uint32_t head_dim)
    {
        const char* base = (const char*)(data + first * stride);
        const uint32_t bytes = (uint32_t)stride * sizeof(T), most = last - first, lds = lds_address(tile) + wave_id() * kWave * 16;
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
            const uint32_t at = s * kThreads + threadIdx.x, row = at / kPieces, piece = (at % kPieces) ^ turn_of<kD>(row);
            if (kFull || piece * 8 < head_dim) memory_to_lds(lds + s * kThreads * 16, base, umin(row, most) * bytes + piece * 16);
        }
    }
};

// kN products whose A operands come from LDS: `read(i)` of one is under way while kAhead others are made of `multiply(i, operand)`.  The compiler
// keeps this order (other instructions may move): left to itself it waits for every operand right behind its read.
//
// kPriority: the wave's while it makes them.  With 1 a wave that has products to make goes before the one beside it that makes weights: both passes of one sequence of 4096 with 32
// heads of 128 take 601 us instead of 627 with it in the backward kernels; the forward kernel, whose tiles are twice as long, is 0.7 % slower with it and goes without.
template <int kN, int kAhead, typename T, int kPriority = 0, typename Read, typename Multiply> __device__ __forceinline__ void products(Read read, Multiply multiply)
{
    V8<T> a[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) a[i] = read(i);
    __builtin_amdgcn_sched_barrier(kOthersMayMove);
    if (kPriority) __builtin_amdgcn_s_setprio(kPriority);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        multiply(i, a[i % kAhead]);
        if (i + kAhead < kN) a[i % kAhead] = read(i + kAhead);
        __builtin_amdgcn_sched_barrier(kOthersMayMove);
    }
    if (kPriority) __builtin_amdgcn_s_setprio(0);
}

// The tiles that the wave's accesses were asked for before the last `kLater` ones have landed, its own reads are done, and so are the other
// waves': behind this the tile may be read, and the one read before it written.
template <int kLater> __device__ __forceinline__ void tiles_landed()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLater) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int kWords, int kThreads> __device__ __forceinline__ void clear_lds(void* lds)
{
    for (int i = threadIdx.x; i < kWords / 4; i += kThreads) ((uint4*)lds)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
}

// One row per lane (row l % 32 of a tile) as the operand of products over the columns: step c holds columns 16 c + 8 (l / 32) .. + 7.
template <typename T, int kD, bool kFull> __device__ __forceinline__ void load_row(V8<T> (&v)[kD / 16], const T* row, uint32_t head_dim)
{
    const uint32_t half = lane_id() >> 5;
#pragma unroll
    for (int c = 0; c < kD / 16; ++c) {
        const uint32_t col = 16 * c + 8 * half;
        if (kFull || col < head_dim) v[c] = *(const V8<T>*)(row + col);
        else v[c] = V8<T>{};
    }
}

// A result tile [columns of a head, in tiles of 32][rows] to memory: the lane's row, four neighbouring columns at a time.
template <typename T, int kD, bool kFull> __device__ __forceinline__ void store_row(T* row, const f32x16 (&x)[kD / 32], float factor, uint32_t head_dim)
{
    const uint32_t half = lane_id() >> 5;
#pragma unroll
    for (int d = 0; d < kD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t col = 32 * d + 8 * i + 4 * half;
            typedef float f32x4 __attribute__((ext_vector_type(4)));
            const f32x4 v = {x[d][4 * i] * factor, x[d][4 * i + 1] * factor, x[d][4 * i + 2] * factor, x[d][4 * i + 3] * factor};
            if (kFull || col < head_dim) *(V4<T>*)(row + col) = __builtin_convertvector(v, V4<T>);
        }
}

// Where a row does not see a key its weight is 0, but 0 times an infinity or a NaN in what the key stands for is none: in the tiles on a piece's diagonal these
// would reach rows that do not see them.  So a wave whose results are not all finite makes them once more, pair by pair in 32 bits, without the
// pairs that are masked (rows_again, keys_again).  The check is 64 instructions a wave, less than 1 % of one sequence of 8192.
template <int kN> __device__ __forceinline__ bool not_finite(const f32x16 (&x)[kN])
{
    float t[4] = {};
#pragma unroll
    for (int d = 0; d < kN; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i % 4] = __builtin_fmaf(x[d][i], 0.f, t[i % 4]);
    return (t[0] + t[1]) + (t[2] + t[3]) != 0.f;
}

// Whether nothing can change the lane's results any more: then the pairs that are left need not be looked at (a step whose gradients have all overflowed is one of these).
// (A maximum is NaN only if everything is.)
template <int kN> __device__ __forceinline__ bool all_nan(const f32x16 (&x)[kN], uint32_t head_dim)
{
    float most = as_float(0x7fc00000u);
    const uint32_t half = kept(lane_id() >> 5);
#pragma unroll
    for (int d = 0; d < kN; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (32 * d + 8 * i + 4 * half < head_dim) most = max3(max3(most, x[d][4 * i], x[d][4 * i + 1]), x[d][4 * i + 2], x[d][4 * i + 3]);
    return most != most;
}

// Scalar product of the lane's row (as load_row gives it, half of its columns; the other half is across) and a row in memory.
template <typename T, int kD, bool kFull> __device__ __forceinline__ float dot_row(const V8<T> (&v)[kD / 16], const T* row, uint32_t head_dim)
{
    float sum = 0.f;
    const uint32_t half = kept(lane_id() >> 5);
#pragma unroll
    for (int c = 0; c < kD / 16; ++c) {
        const uint32_t col = 16 * c + 8 * half;
        if (kFull || col < head_dim) sum += dot(__builtin_convertvector(v[c], f32x8), load8(row + col));
        __builtin_amdgcn_sched_barrier(0);                   // (one piece of the row in registers at a time: the walks above have none to spare)
    }
    return sum + across(sum);
}

// A row's running maximum (of unscaled scores) while none was seen: below every finite score there is.
constexpr float kNoScore = -3.402823466e38f;

// Maximum and sum of 2^(scale (s - maximum)) of the scores of the lane's row (q as load_row gives it) with keys from .. to - 1 that it sees, key by key.  The scores are those that
// the pair-by-pair walks make, to the last bit, whichever of the two rows is in registers: where they are huge, one that is rounded otherwise would be worlds away.
template <typename T, int kD, bool kFull>
__device__ __forceinline__ f32x2 row_stats(const V8<T> (&q)[kD / 16], const T* k, uint64_t stride, uint32_t from, uint32_t to, uint32_t row, float scale, uint32_t head_dim)
{
    float m = kNoScore, total = 0.f;
#pragma unroll 1
    for (uint32_t key = from; key < to; ++key) {
        const float s = dot_row<T, kD, kFull>(q, k + key * stride, head_dim);
        if (key > row) continue;
        const float raised = fmaxf(m, s);
        total = total * exp2_fast((m - raised) * scale) + exp2_fast((s - raised) * scale);
        m = raised;
    }
    return f32x2{m, total};
}

// x += w * (a row in memory), columns as store_row has them.
template <typename T, int kD, bool kFull> __device__ __forceinline__ void add_row(f32x16 (&x)[kD / 32], float w, const T* row, uint32_t head_dim)
{
    const uint32_t half = kept(lane_id() >> 5);
#pragma unroll
    for (int d = 0; d < kD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t col = 32 * d + 8 * i + 4 * half;
            if (!kFull && col >= head_dim) continue;
            const V4<T> v = *(const V4<T>*)(row + col);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[d][4 * i + j] = __builtin_fmaf(w, (float)v[j], x[d][4 * i + j]);
            __builtin_amdgcn_sched_barrier(0);
        }
}

// Tensor of a call: numbers, and strides between tokens and heads.
template <typename T> struct Heads {
    T* data;
    uint64_t token, head;
    __device__ __forceinline__ T* at(uint64_t t, uint32_t h) const { return data + t * token + h * head; }
};

constexpr int kPieceRows = 128;                              // four waves of 32

// kRows rows of one sequence, or of the padding behind the last one (no_keys).
struct Piece {
    uint32_t begin, end;                                     // the sequence
    uint32_t first;                                          // first row of the piece; first >= end: nothing to do
    bool no_keys;
};

// The `index`-th piece of the packed batch, every sequence cut into pieces of kRows rows from its beginning.  Sequences are counted through 64
// at a time; boundaries are held to the batch, whatever they say, so that nothing is read or written outside of it.
template <int kRows> __device__ __forceinline__ Piece find_piece(const uint32_t* __restrict__ bounds, uint32_t sequences, uint32_t tokens, uint32_t index)
{
    uint32_t before = 0;
    for (uint32_t s = 0; s < sequences; s += kWave) {
        const uint32_t i = s + lane_id();
        uint32_t lo = 0, hi = 0;
        if (i < sequences) {
            lo = umin(bounds[i], tokens);
            hi = umax(lo, umin(bounds[i + 1], tokens));
        }
        const uint32_t n = (hi - lo + kRows - 1) / kRows, upto = wave_scan_add(n), total = read_lane(upto, kWave - 1);
        if (index - before < total) {
            const int at = __builtin_ctzll(__ballot(upto > index - before));
            const uint32_t from = before + read_lane(upto, at) - read_lane(n, at);
            const uint32_t begin = read_lane(lo, at);
            return {begin, read_lane(hi, at), begin + (index - from) * kRows, false};
        }
        before += total;
    }
    const uint32_t end = uniform(umin(bounds[sequences], tokens));
    const uint64_t first = end + (uint64_t)(index - before) * kRows;
    return {end, tokens, first < tokens ? (uint32_t)first : tokens, true};
}

// How many pieces a batch can have at most.
inline uint64_t most_pieces(uint32_t tokens, uint32_t sequences, uint32_t rows) { return (uint64_t)tokens / rows + sequences + 1; }

// What the workgroups of a kernel share out among themselves: pieces of every head, and (dk and dv) parts of the walk over a piece's rows.
//
// The longest walks come first, those of all heads: the last workgroups to begin are then the shortest.  (Heads one after the other instead, each from
// its longest walk on, took 198 us for one sequence of 4096 and 32 heads of 128, this order takes 156.)  For a single sequence the order of the pieces is
// known; for several, attention_list makes a list of all pieces in that order.  Without one (a single sequence; calls that would be over before the list is
// made) every workgroup counts through the boundaries itself.
struct Work {
    const uint4* list;                                       // {begin, end, rank, no_keys}; rank: the piece's number from that end of its sequence
    const uint32_t* bounds;                                  //   whose walk is shortest
    uint32_t sequences, tokens, pieces, heads, parts;
};

struct Task {
    uint32_t head, part;
    Piece piece;
};

// kFromEnd: a piece's walk is the longer the nearer it is to the end of its sequence (rows; else keys: to the beginning).
template <int kRows, bool kFromEnd> __device__ __forceinline__ Task take_task(const Work& w)
{
    // Workgroups go to the 8 dies in turn: neighbouring heads (which may share keys) to the same die.
    const uint32_t at = blockIdx.x % w.heads, rest = blockIdx.x / w.heads, head = w.heads % 8 == 0 ? at % 8 * (w.heads / 8) + at / 8 : at, piece = rest / w.parts;
    if (w.list) {
        const uint4 e = w.list[piece];
        const uint32_t begin = uniform(e.x), end = uniform(e.y), rank = uniform(e.z), n = (end - begin + kRows - 1) / kRows;
        return {head, rest % w.parts, {begin, end, begin + (kFromEnd ? rank : n - 1 - rank) * kRows, uniform(e.w) != 0}};
    }
    return {head, rest % w.parts, find_piece<kRows>(w.bounds, w.sequences, w.tokens, kFromEnd ? w.pieces - 1 - piece : piece)};
}

// Into how many parts the walks are cut, for kernels whose pieces alone do not give every CU two workgroups: parts of `least` steps or more (of a walk of
// average length; `steps`: those of the longest walk in a sequence of average length), `most` at most.  A part leaves its sums in the workspace, and a
// kernel of its own adds them up.
inline uint32_t parts_of(uint64_t workgroups, uint64_t steps, uint32_t least, uint32_t most)
{
    uint64_t parts = workgroups >= 512 ? 1 : (512 + workgroups - 1) / workgroups;
    if (parts > steps / (2 * least)) parts = steps / (2 * least);
    return parts < 1 ? 1 : parts > most ? most : (uint32_t)parts;
}
inline uint64_t average_rows(const stalloc_attention_shape* s) { return ((uint64_t)s->tokens + s->sequences - 1) / s->sequences; }
inline uint64_t row_pieces(const stalloc_attention_shape* s) { return ((uint64_t)s->tokens + kPieceRows - 1) / kPieceRows; }

// A list pays where the workgroups do not all run at once and sequences differ.
inline bool list_pays(uint64_t workgroups, uint32_t sequences) { return sequences > 1 && workgroups >= 2048; }

void launch_attention_list(const uint32_t* bounds, uint32_t sequences, uint32_t tokens, uint32_t pieces, uint4* list, uint32_t* status, hipStream_t stream);

// One workgroup's look at all boundaries; whether they are as they should be.
__device__ __forceinline__ bool check_bounds(const uint32_t* __restrict__ bounds, uint32_t sequences, uint32_t tokens, uint32_t* status)
{
    __shared__ uint32_t bad;
    if (threadIdx.x == 0) bad = bounds[0] != 0;
    __syncthreads();
    bool wrong = false;
    for (uint32_t i = threadIdx.x; i < sequences; i += blockDim.x) wrong |= bounds[i] > bounds[i + 1] || bounds[i + 1] > tokens;
    if (wrong) bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) *status = bad ? STALLOC_ERR_BAD_BOUNDS : STALLOC_OK;
    return !bad;
}

constexpr uint64_t kMostStride = 1u << 24;

inline bool shape_ok(const stalloc_attention_shape* s)
{
    return s && (s->dtype == STALLOC_BF16 || s->dtype == STALLOC_F16) && s->tokens >= 1 && s->tokens < 0x80000000u && s->sequences >= 1 &&
           s->sequences < 0x80000000u && s->kv_heads >= 1 && s->heads >= s->kv_heads && s->heads % s->kv_heads == 0 && s->heads < 0x10000u &&
           s->head_dim >= 8 && s->head_dim <= 128 && s->head_dim % 8 == 0 && s->scale > 0.f && s->scale < 1e8f;
}

inline bool heads_ok(const stalloc_heads* t, const stalloc_attention_shape* s, uint32_t heads, bool written)
{
    if (!t || !t->data || !aligned(t->data, 16) || t->token_stride % 8 || t->head_stride % 8) return false;
    if (t->token_stride > kMostStride || t->head_stride >> 40) return false;     // (offsets inside a tile have 32 bits)
    return !written || ((s->tokens == 1 || t->token_stride >= s->head_dim) && (heads == 1 || t->head_stride >= s->head_dim));
}

template <typename T> inline Heads<T> heads_of(const stalloc_heads* t) { return {static_cast<T*>(t->data), t->token_stride, t->head_stride}; }

}  // namespace stalloc
