// Products of rows with weights of 4 bits, and the gradient of those rows.
//
//   y[m, n] = sum over k of x[m, k] W[n, k] + b[n],   grad_x[m, k] = sum over n of grad_y[m, n] W[n, k]
//   W[n, k] = zero[n, g] + step[n, g] code[n, k],  g = k div group
//
// A word holds eight codes of neighbouring k, pair i of them in bits 4 i and 16 + 4 i, so that a shift and a mask leave a pair in the halves of a register.
// As the upper four bits of a fraction, under the exponent of 2^-8 (bfloat16) or 2^-14 (binary16), that is a pair of numbers 1 + code / 16 times that power: the matrix
// instructions multiply both exactly.  So a group's sum of x code is a sum of exact products in binary32, to which step, and zero times the group's sum of
// x (one more product, with a constant), come afterwards.  A binary32 x goes as the three bfloat16 numbers that make up x / 2048, and its codes as converted numbers:
// sums of 16 x beside those of x code would cost it 2 of its 24 bits.  All of these are so small that no group's sum is larger than its largest x, and none of
// finite x overflows; the total is kept in their unit until the end.
//
// Measured on one MI355X, whose copy of 1 GiB reaches 5.1 TB/s and whose library product of 8192^3 1.21 PFLOP/s in bfloat16, from the host, calls one behind the other (a
// profiler's trace, which lets no kernel begin before the last has ended, shows up to 0.9 us more for each): one row of 4096 x 4096 in groups of 128
// 4.9 us, 23 rows of 8192 x 16384 in binary16 and groups of 64 26 us (3.0 TB/s), 4096 rows of 8192 x 8192 in bfloat16 555 us (990 TFLOP/s), the gradient of 2047 rows of
// 4096 inputs and 8192 outputs 214 us (640 TFLOP/s).
#include "actq_heads.h"

namespace actq {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// How a type of x meets the codes.  With sums of x (binary32: kSum x) times what stands for its code, and times a plain number (a pair of it: kPlain), which are sums of kSum x,
// zero x + step x code = kBack (step sum + (kZero zero - kShift step) plain).
template <typename T>
struct Meets;
template <>
struct Meets<__bf16> {
    typedef bf16x8 vector;
    static constexpr uint32_t kPlain = 0x3b803b80u;   // 2^-8, and what lies under a code
    static constexpr int kCodeBit = 3;
    static constexpr float kSum = 0x1p-8f, kZero = 0x1p-4f, kShift = 1.0f, kBack = 0x1p12f;
};
template <>
struct Meets<_Float16> {
    typedef f16x8 vector;
    static constexpr uint32_t kPlain = 0x04000400u;   // 2^-14, the smallest with all its bits: sums of products with subnormal numbers are less exact
    static constexpr int kCodeBit = 6;
    static constexpr float kSum = 0x1p-14f, kZero = 0x1p-4f, kShift = 1.0f, kBack = 0x1p18f;
};
template <>
struct Meets<float> {
    typedef bf16x8 vector;
    static constexpr uint32_t kPlain = 0x3f803f80u;   // 1
    static constexpr float kSum = 0x1p-11f, kZero = 1.0f, kShift = 0.0f, kBack = 0x1p11f;
};

template <typename T>
constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;

// The eight codes of a word in the order of their k.
template <typename T>
__device__ __forceinline__ typename Meets<T>::vector codes_of(uint32_t w)
{
    u32x4 v;
    if constexpr (sizeof(T) == 2) {
        constexpr int kBit = Meets<T>::kCodeBit;
        uint32_t under = Meets<T>::kPlain;
        asm("" : "+v"(under));   // in a vector register: one instruction takes one constant from elsewhere, and so masks and sets at once
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ((4 * i < kBit ? w << (kBit - 4 * i) : w >> (4 * i - kBit)) & 0x000f000fu << kBit) | under;
    } else {
        const uint32_t half[2] = {w & 0x0f0f0f0fu, w >> 4 & 0x0f0f0f0fu};   // bytes of the codes 0, 4, 1, 5 and 2, 6, 3, 7
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float low = static_cast<float>(half[i % 2] >> 8 * (i / 2) & 255u), high = static_cast<float>(half[i % 2] >> 8 * (i / 2 + 2) & 255u);
            v[i] = __builtin_bit_cast(uint32_t, low) >> 16 | __builtin_bit_cast(uint32_t, high);   // whole numbers up to 15 end in zeros
        }
    }
    return __builtin_bit_cast(typename Meets<T>::vector, v);
}

// Eight values of x as vectors for the matrix instructions.  Binary32, times kSum: the upper 8 bits of a value's 24, of the rest, and what is left, each of them a
// bfloat16 number.
template <typename T>
__device__ __forceinline__ void pieces_of(const Eight<T>& e, typename Meets<T>::vector (&v)[kPieces<T>])
{
    if constexpr (sizeof(T) == 2) {
        v[0] = e.v;
    } else {
        u32x4 p[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t bits[3][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float x = Meets<T>::kSum * e.v[2 * i + j];
                bits[0][j] = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
                const float rest = x - __builtin_bit_cast(float, bits[0][j]);
                bits[1][j] = __builtin_bit_cast(uint32_t, rest) & 0xffff0000u;
                bits[2][j] = __builtin_bit_cast(uint32_t, rest - __builtin_bit_cast(float, bits[1][j]));
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) p[k][i] = bits[k][0] >> 16 | (bits[k][1] & 0xffff0000u);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) v[k] = __builtin_bit_cast(bf16x8, p[k]);
    }
}

template <int N>
__device__ __forceinline__ void split(float v, uint32_t (&bits)[N])   // bfloat16 numbers in the upper halves whose sum is v, but for what a last one leaves
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        bits[i] = __builtin_bit_cast(uint32_t, v);
        if (i == N - 1) bits[i] += 0x7fffu + (bits[i] >> 16 & 1u);   // to nearest: what is left of 24 bits is exact, of 16 it is not
        bits[i] &= 0xffff0000u;
        v -= __builtin_bit_cast(float, bits[i]);
    }
}

__device__ __forceinline__ float zero_of(uint32_t header) { return __builtin_bit_cast(float, header << 16); }
__device__ __forceinline__ float step_of(uint32_t header) { return __builtin_bit_cast(float, header & 0xffff0000u); }

// What a group's plain sum is multiplied by.
template <typename T>
__device__ __forceinline__ float plain_factor(uint32_t header)
{
    return fmaf(-Meets<T>::kShift, step_of(header), Meets<T>::kZero * zero_of(header));
}

struct Weights4 {
    const uint32_t* codes;    // [outputs, groups * group / 8]
    const uint32_t* header;   // [outputs, groups]: zero in the lower half, step in the upper one
    int32_t inputs, outputs, groups;
};

Weights4 weights_of(const actq_weights4* w)
{
    return {w->codes, reinterpret_cast<const uint32_t*>(w->header), w->inputs, w->outputs, (w->inputs + w->group - 1) / w->group};
}

template <typename T>
__device__ __forceinline__ float bias_of(const void* bias, int wide, int n)
{
    if (!bias) return 0.0f;
    return wide ? static_cast<const float*>(bias)[n] : static_cast<float>(static_cast<const T*>(bias)[n]);
}

// The parts of a sum over a long axis, joined in their order.
template <typename T>
__global__ __launch_bounds__(256) void linear4_join_kernel(const float* parts, int32_t count, int64_t rows, int32_t columns, const void* bias, int wide_bias, T* out, int64_t stride)
{
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, all = rows * columns;
    if (unit >= all) return;
    const int64_t m = unit / columns;
    const int n = static_cast<int>(unit - m * columns);
    float sum = bias_of<T>(bias, wide_bias, n);
    for (int i = 0; i < count; i += 8) {
        float v[8];   // all in flight
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j < count ? parts[(i + j) * all + unit] : 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[j];
    }
    out[m * stride + n] = static_cast<T>(sum);
}

// ----------------------------------------------------------------------------- few rows

// 16 rows and COLUMNS x 16 outputs a workgroup, whose wavefronts take spans of 128 k in turn: for one token of a small matrix every compute unit has 16 wavefronts
// with all that they need on its way at once.  A lane's codes of a group are neighbours (a quarter of the group), and so are its x.  What bounds it: the chain of trips to
// memory, and the loads of x, of which it makes as many for a row as for 16.
template <typename T>
struct FewArgs {
    Weights4 w;
    const T* x;
    int64_t x_stride;
    const void* bias;
    int32_t wide_bias;
    T* y;
    int64_t y_stride;
    int64_t rows;
};

constexpr int kSpan = 128;

template <typename T, int GROUP, int COLUMNS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear4_few_kernel(FewArgs<T> a)
{
    constexpr int kGroups = kSpan / GROUP, kWords = GROUP / 32;   // of a span; of a lane and group
    typedef typename Meets<T>::vector V;
    typedef uint32_t words __attribute__((ext_vector_type(kWords), aligned(4)));
    typedef uint32_t headers __attribute__((ext_vector_type(kGroups), aligned(4)));
    __shared__ float joined[WAVES][COLUMNS][256];
    const int lane = threadIdx.x % 64, at = lane % 16, quarter = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t first_row = static_cast<int64_t>(blockIdx.y) * 16;
    const int first_column = blockIdx.x * (16 * COLUMNS);
    const int row_words = a.w.groups * (GROUP / 8);
    const uint32_t* codes[COLUMNS];
    const uint32_t* header[COLUMNS];
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c) {
        const int64_t n = min(first_column + 16 * c + at, a.w.outputs - 1);
        codes[c] = a.w.codes + n * row_words;
        header[c] = a.w.header + n * a.w.groups;
    }
    const T* const x = a.x + min(first_row + at, a.rows - 1) * a.x_stride;
    const V plainly = __builtin_bit_cast(V, u32x4{Meets<T>::kPlain, Meets<T>::kPlain, Meets<T>::kPlain, Meets<T>::kPlain});
    f32x4 total[COLUMNS] = {};

    // what a span needs; that of the wavefront's next one is on its way while this one is worked on
    struct Span {
        words word[COLUMNS][kGroups];
        headers head[COLUMNS];
        Eight<T> x[kGroups * kWords];
    };
    const auto load = [&](Span& s, int span) {
        const int group = span * kGroups;
        if (group + kGroups <= a.w.groups) {
#pragma unroll
            for (int c = 0; c < COLUMNS; ++c) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) s.word[c][g] = *reinterpret_cast<const words*>(codes[c] + (group + g) * (GROUP / 8) + quarter * kWords);
                s.head[c] = *reinterpret_cast<const headers*>(header[c] + group);
            }
        } else {   // groups that are none stand for zeros
#pragma unroll
            for (int c = 0; c < COLUMNS; ++c)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const bool there = group + g < a.w.groups;
                    s.word[c][g] = *reinterpret_cast<const words*>(codes[c] + (there ? group + g : 0) * (GROUP / 8) + quarter * kWords);
                    s.head[c][g] = there ? header[c][group + g] : 0u;
                }
        }
        if ((span + 1) * kSpan <= a.w.inputs) {
#pragma unroll
            for (int j = 0; j < kGroups * kWords; ++j) s.x[j].load(x + span * kSpan + j / kWords * GROUP + quarter * (GROUP / 4) + 8 * (j % kWords));
        } else {
#pragma unroll
            for (int j = 0; j < kGroups * kWords; ++j) {
                const int k = span * kSpan + j / kWords * GROUP + quarter * (GROUP / 4) + 8 * (j % kWords);
#pragma unroll
                for (int i = 0; i < 8; ++i) s.x[j].v[i] = k + i < a.w.inputs ? x[k + i] : static_cast<T>(0.0f);
            }
        }
    };
    const int spans = (a.w.inputs + kSpan - 1) / kSpan;
    Span now;
    if (wave < spans) load(now, wave);
    for (int span = wave; span < spans; span += WAVES) {
        Span next;
        if (span + WAVES < spans) load(next, span + WAVES);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            f32x4 sum[COLUMNS] = {}, plain = {};
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                V code[COLUMNS];
#pragma unroll
                for (int c = 0; c < COLUMNS; ++c) code[c] = codes_of<T>(kWords == 1 ? now.word[c][g][0] : now.word[c][g][j]);
                V p[kPieces<T>];
                pieces_of<T>(now.x[g * kWords + j], p);
#pragma unroll
                for (int i = kPieces<T> - 1; i >= 0; --i) {
                    plain = multiply(p[i], plainly, plain);
#pragma unroll
                    for (int c = 0; c < COLUMNS; ++c) sum[c] = multiply(p[i], code[c], sum[c]);
                }
            }
#pragma unroll
            for (int c = 0; c < COLUMNS; ++c) {
                const uint32_t head = now.head[c][g];
                const float step = step_of(head), factor = plain_factor<T>(head);
#pragma unroll
                for (int i = 0; i < 4; ++i) total[c][i] = fmaf(factor, plain[i], fmaf(step, sum[c][i], total[c][i]));
            }
        }
        now = next;
    }
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) joined[wave][c][(4 * quarter + i) * 16 + at] = total[c][i];
    __syncthreads();
    for (int i = threadIdx.x; i < COLUMNS * 256; i += 64 * WAVES) {
        const int column = i % (16 * COLUMNS), row = i / (16 * COLUMNS), tile = column / 16, place = row * 16 + column % 16;
        const int64_t m = first_row + row;
        const int n = first_column + column;
        if (m >= a.rows || n >= a.w.outputs) continue;
        float sum = joined[0][tile][place];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += joined[w][tile][place];
        a.y[m * a.y_stride + n] = static_cast<T>(fmaf(sum, Meets<T>::kBack, bias_of<T>(a.bias, a.wide_bias, n)));
    }
}

// ----------------------------------------------------------------------------- many rows

// What x looks like for the kernel below: 16-bit numbers, whole spans of k, zeros beyond the last input.  16-bit rows that are like that already are taken
// as they lie; others are copied (binary32: split into the bfloat16 numbers that make it up).  Beside it the plain sums of every group of a row, as
// three bfloat16 numbers each.
template <typename T>
struct PrepareArgs {
    const T* x;
    int64_t stride;
    int32_t inputs, padded;   // whole spans
    int64_t rows, first;      // first: workgroups of earlier launches
    u32x4* copy;              // [pieces][rows][padded / 8]; null: none
    u32x2* sums;              // [padded / group][rows]
};

template <typename T, int GROUP>
__global__ __launch_bounds__(256) void linear4_prepare_kernel(PrepareArgs<T> a)
{
    const int chunks = a.padded / 8;
    const int64_t unit = (a.first + blockIdx.x) * 256 + threadIdx.x;
    const bool there = unit < a.rows * chunks;
    const int64_t m = there ? unit / chunks : 0;
    const int chunk = there ? static_cast<int>(unit - m * chunks) : 0, k = 8 * chunk;
    const T* const x = a.x + m * a.stride + k;
    Eight<T> e;
    if (k + kLaneValues <= a.inputs) {
        e.load(x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = k + i < a.inputs ? x[i] : static_cast<T>(0.0f);
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(static_cast<float>(e.v[i]), Meets<T>::kSum, sum);
#pragma unroll
    for (int step = 1; step < GROUP / 8; step *= 2) sum += __shfl_xor(sum, step);
    if (!there) return;
    if (a.copy) {
        typename Meets<T>::vector p[kPieces<T>];
        pieces_of<T>(e, p);
#pragma unroll
        for (int i = 0; i < kPieces<T>; ++i) a.copy[(i * a.rows + m) * chunks + chunk] = __builtin_bit_cast(u32x4, p[i]);
    }
    if (chunk % (GROUP / 8) != 0) return;
    uint32_t bits[3];
    split(sum, bits);
    a.sums[chunk / (GROUP / 8) * a.rows + m] = u32x2{bits[0] >> 16 | bits[1], bits[2] >> 16};
}

template <typename T>
struct ManyArgs {
    Weights4 w;
    const uint16_t* x;        // [pieces][rows][x_stride], 16-byte aligned rows
    int64_t x_stride, x_piece;
    const u32x2* sums;
    int32_t padded;
    const void* bias;
    int32_t wide_bias;
    T* y;
    int64_t y_stride;
    int64_t rows;
    int32_t row_tiles, column_tiles;
    int32_t share;            // k of a part; whole spans
    float* parts;             // [parts][rows][outputs]; null: the only part writes y
};

// Sixteen or four bytes of every lane from memory to neighbouring places in the LDS, `to` being the first lane's, without registers between.
typedef const __attribute__((address_space(1))) void* InMemory;
typedef __attribute__((address_space(3))) void* InLds;

__device__ __forceinline__ void to_lds(const void* from, u32x4* to) { __builtin_amdgcn_global_load_lds((InMemory) reinterpret_cast<uintptr_t>(from), (InLds)to, 16, 0, 0); }
__device__ __forceinline__ void to_lds(const void* from, uint32_t* to) { __builtin_amdgcn_global_load_lds((InMemory) reinterpret_cast<uintptr_t>(from), (InLds)to, 4, 0, 0); }

// Until all but the last COUNT of a wavefront's loads have arrived, in all wavefronts of the workgroup.
template <int COUNT>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COUNT) : "memory");
}

// A workgroup's tile is ROWS rows x 256 outputs, made of blocks of 32 x 32: 128 rows, two by two blocks a wavefront, or 32, one.  A group's sums of products
// and the total are both what ordinary instructions work with, so they share the 256 registers that these see, and 128 rows take two wavefronts a SIMD.  x, codes and headers
// go from memory to the LDS without registers, two stages of 128 k ahead (binary32, three times the bytes: one of 64 with 128 rows; four stages ahead under 32 rows give nothing); a wavefront turns the codes of its outputs
// into numbers in registers.  Under 32 rows, where memory is what counts, the groups' plain sums of x are one more product.
template <typename T, int GROUP, int ROWS>
__global__ __launch_bounds__(512, 2) void linear4_many_kernel(ManyArgs<T> a)
{
    typedef typename Meets<T>::vector V;
    constexpr int kP = kPieces<T>, kB = ROWS == 128 ? 2 : 1, kRing = kP == 1 || kB == 1 ? 3 : 2, kDepth = kP == 1 ? 128 : 64, kRows = ROWS, kColumns = 256;
    constexpr int kChunks = kDepth / 8, kSlots = kDepth / 32;   // 16 bytes of a row of x, of an output's codes
    constexpr int kScaled = GROUP < kDepth ? GROUP : kDepth, kHeads = kDepth / kScaled, kSteps = kScaled / 16;
    constexpr int kMoves = kRows * kChunks >= 512 ? kRows * kChunks / 512 : 1, kCodeMoves = kColumns * kSlots / 512;
    constexpr int kLoads = kP * kMoves + kCodeMoves;   // of a wavefront and stage, beside headers
    constexpr int kHeadGroups = 8;                     // headers of so many groups are fetched at a time: one by one they would take as many lines of the caches as the codes
    // one array: of several the compiler knows which of them a load to the LDS writes, and waits for it before the next read of that one
    constexpr int kTilePlace = kRows * kChunks < 512 ? 512 : kRows * kChunks, kCodes = kP * kTilePlace, kStage = kCodes + kColumns * kSlots, kHeadPlace = kColumns * kHeadGroups;
    // as many places for headers as the stages on their way can need beside the one that is worked on
    constexpr int kHeadStages = kHeadGroups * GROUP / kDepth, kHeadPlaces = 1 + (kRing - 1 + kHeadStages - 1) / kHeadStages;
    __shared__ u32x4 lds[kRing * kStage + kHeadPlaces * kHeadPlace / 4];
    uint32_t* const heads = reinterpret_cast<uint32_t*>(lds + kRing * kStage);   // [kHeadPlaces][outputs][kHeadGroups]
    const int lane = threadIdx.x % 64, at = lane % 32, half = lane / 32;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    // each XCD (workgroups go to them in turn) takes a run of tiles, bands of 4 row tiles through all column tiles: their rows and codes stay in its L2
    const int tiles = a.row_tiles * a.column_tiles, share = (tiles + 7) / 8, unit = blockIdx.x % 8 * share + blockIdx.x / 8;
    if (unit >= tiles || static_cast<int>(blockIdx.x / 8) >= share) return;
    const int band = unit / (4 * a.column_tiles), in_band = unit - band * 4 * a.column_tiles, high = min(4, a.row_tiles - 4 * band);
    const int64_t first_row = static_cast<int64_t>(4 * band + in_band % high) * kRows;
    const int first_column = (in_band / high) * kColumns, row_words = a.w.groups * (GROUP / 8);
    const auto code_swizzle = [](int column) { return kSlots == 4 ? column >> 2 & 3 : 0; };

    // where the lane's loads come from: the place in the LDS goes by the lane, so what lies there is chosen here
    const uint16_t* x_from[kMoves];
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
        const int row = (i * 512 + threadIdx.x) / kChunks % kRows, chunk = threadIdx.x % kChunks ^ (row & (kChunks - 1));
        const int64_t m = first_row + row;
        x_from[i] = a.x + (m < a.rows ? m : a.rows - 1) * a.x_stride + 8 * chunk;
    }
    const uint32_t* codes_from[kCodeMoves];
    int code_chunk[kCodeMoves];
#pragma unroll
    for (int i = 0; i < kCodeMoves; ++i) {
        const int column = (i * 512 + threadIdx.x) / kSlots;
        const int64_t n = min(first_column + column, a.w.outputs - 1);
        codes_from[i] = a.w.codes + n * row_words;
        code_chunk[i] = threadIdx.x % kSlots ^ code_swizzle(column);
    }
    const int begin = blockIdx.y * a.share, end = min(begin + a.share, a.padded);   // the part's k
    const auto load = [&](int k, int to) {
#pragma unroll
        for (int p = 0; p < kP; ++p)
#pragma unroll
            for (int i = 0; i < kMoves; ++i) to_lds(x_from[i] + p * a.x_piece + k, lds + to * kStage + p * kTilePlace + i * 512 + wave * 64);
        // beyond the last group x is zero, whatever the codes are
#pragma unroll
        for (int i = 0; i < kCodeMoves; ++i) to_lds(codes_from[i] + 4 * min(k / 32 + code_chunk[i], row_words / 4 - 1), lds + to * kStage + kCodes + i * 512 + wave * 64);
        if ((k - begin) % (kHeadGroups * GROUP) != 0) return;
        const int place = (k - begin) / (kHeadGroups * GROUP) % kHeadPlaces, group = min(k / GROUP + static_cast<int>(threadIdx.x % kHeadGroups), a.w.groups - 1);
#pragma unroll
        for (int i = 0; i < kHeadPlace / 512; ++i) {
            const int64_t n = min(first_column + (i * 512 + static_cast<int>(threadIdx.x)) / kHeadGroups, a.w.outputs - 1);
            to_lds(a.w.header + n * a.w.groups + group, heads + place * kHeadPlace + i * 512 + wave * 64);
        }
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i)
        if (begin + i * kDepth < end) load(begin + i * kDepth, i);

    // the factors' two terms times the groups' plain sums: products of the parts of both.  A lane takes four neighbouring groups at a time.
    const int columns = kB == 2 ? wave % 4 * 64 : wave * 32, rows = kB == 2 ? wave / 4 * 64 : 0;   // the wavefront's place in the tile
    f32x16 total[kB][kB] = {};
    if constexpr (kB == 2) {
        const u32x2* sums[2];
        const uint32_t* header[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t m = first_row + rows + 32 * r + at;
            sums[r] = a.sums + (m < a.rows ? m : a.rows - 1);
            header[r] = a.w.header + static_cast<int64_t>(min(first_column + columns + 32 * r + at, a.w.outputs - 1)) * a.w.groups;
        }
        constexpr int kTogether = Meets<T>::kShift != 0.0f ? 1 : 2;   // groups of a lane in a product
        const int groups = min(end / GROUP, a.w.groups);
        for (int g = begin / GROUP; g < groups; g += 8) {
            const int mine = g + 4 * half;
            u32x2 v[2][4];
            u32x4 h[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (g + 8 <= groups) {
                    typedef u32x4 any __attribute__((aligned(4)));
                    h[r] = *reinterpret_cast<const any*>(header[r] + mine);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[r][j] = mine + j < groups ? header[r][mine + j] : 0u;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) v[r][j] = sums[r][min(mine + j, groups - 1) * a.rows];
            }
#pragma unroll
            for (int q = 0; q < 4; q += kTogether) {
                u32x4 s[2], z[2];
#pragma unroll
                for (int j = 0; j < kTogether; ++j) {
                    const uint32_t there = mine + q + j < groups ? ~0u : 0u;   // no NaN times zero
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t head = h[r][q + j], zero = __builtin_bit_cast(uint32_t, Meets<T>::kZero * zero_of(head)) >> 16;
                        s[r][2 * j] = v[r][q + j][0] & there;
                        s[r][2 * j + 1] = v[r][q + j][1] & there;
                        z[r][2 * j] = zero | zero << 16;
                        z[r][2 * j + 1] = zero;
                        if (kTogether == 1) {
                            s[r][2] = s[r][0];
                            s[r][3] = s[r][1];
                            const uint32_t shifted = __builtin_bit_cast(uint32_t, step_of(head) * -Meets<T>::kShift);
                            z[r][2] = shifted | shifted >> 16;
                            z[r][3] = shifted >> 16;
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int c = 0; c < 2; ++c) total[r][c] = multiply(__builtin_bit_cast(bf16x8, s[r]), __builtin_bit_cast(bf16x8, z[c]), total[r][c]);
            }
        }
    }
    const auto place = [](int row, int chunk) { return row * kChunks + (chunk ^ (row & (kChunks - 1))); };
    if (begin + (kRing - 2) * kDepth < end)
        arrived<(kRing - 2) * kLoads>();
    else
        arrived<0>();
    const V plainly = __builtin_bit_cast(V, u32x4{Meets<T>::kPlain, Meets<T>::kPlain, Meets<T>::kPlain, Meets<T>::kPlain});
    int buffer = 0;
    for (int k = begin; k < end; k += kDepth) {
        const int ahead = k + (kRing - 1) * kDepth;
        if (ahead < end) load(ahead, buffer == 0 ? kRing - 1 : buffer - 1);
        const u32x4* const tile = lds + buffer * kStage;
        const u32x4* const codes = tile + kCodes;
        const int group = (k - begin) / GROUP;
#pragma unroll 1   // two groups' sums at once do not fit the registers
        for (int g = 0; g < kHeads; ++g) {
            f32x16 sum[kB][kB], plain;
            uint32_t word[kB][kSteps], head[kB];
#pragma unroll
            for (int c = 0; c < kB; ++c) {
                const int column = columns + 32 * c + at;
                head[c] = heads[(group + g) / kHeadGroups % kHeadPlaces * kHeadPlace + column * kHeadGroups + (group + g) % kHeadGroups];
                if constexpr (GROUP == 32) {   // a group is 16 bytes of an output, a half of them this lane's
                    const u32x2 v = reinterpret_cast<const u32x2*>(&codes[column * kSlots + (g ^ code_swizzle(column))])[half];
                    word[c][0] = v[0];
                    word[c][1] = v[1];
                } else {
#pragma unroll
                    for (int j = 0; j < kSteps / 4; ++j) {
                        const u32x4 v = codes[column * kSlots + ((g * (kScaled / 32) + 2 * j + half) ^ code_swizzle(column))];
#pragma unroll
                        for (int i = 0; i < 4; ++i) word[c][4 * j + i] = v[i];
                    }
                }
            }
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                const int chunk = GROUP == 32 ? 4 * g + 2 * half + step : g * (kScaled / 8) + step / 4 * 8 + 4 * half + step % 4;
                V w[kB];
#pragma unroll
                for (int c = 0; c < kB; ++c) w[c] = codes_of<T>(word[c][step]);
#pragma unroll
                for (int r = 0; r < kB; ++r)
#pragma unroll
                    for (int p = kP - 1; p >= 0; --p) {
                        const V v = __builtin_bit_cast(V, tile[p * kTilePlace + place(rows + 32 * r + at, chunk)]);
                        if constexpr (kB == 1) {
                            if (step == 0 && p == kP - 1) plain = f32x16{};
                            plain = multiply(v, plainly, plain);
                        }
#pragma unroll
                        for (int c = 0; c < kB; ++c) {
                            if (step == 0 && p == kP - 1) sum[r][c] = f32x16{};
                            sum[r][c] = multiply(v, w[c], sum[r][c]);
                        }
                    }
            }
#pragma unroll
            for (int c = 0; c < kB; ++c) {
                const float step = step_of(head[c]), factor = plain_factor<T>(head[c]);
#pragma unroll
                for (int r = 0; r < kB; ++r)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        total[r][c][i] = fmaf(step, sum[r][c][i], total[r][c][i]);
                        if constexpr (kB == 1) total[r][c][i] = fmaf(factor, plain[i], total[r][c][i]);
                    }
            }
        }
        // the next stage; what lies behind it may still be on its way (headers of later groups are waited for)
        if (ahead < end)
            arrived<(kRing - 2) * kLoads>();
        else
            arrived<0>();
        buffer = buffer == kRing - 1 ? 0 : buffer + 1;
    }
#pragma unroll
    for (int c = 0; c < kB; ++c) {
        const int n = first_column + columns + 32 * c + at;
        if (n >= a.w.outputs) continue;
        const int64_t m = first_row + rows + 4 * half;
        if (a.parts) {
            float* const to = a.parts + (blockIdx.y * a.rows + m) * a.w.outputs + n;
#pragma unroll
            for (int r = 0; r < kB; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int down = 32 * r + 8 * (i / 4) + i % 4;
                    if (m + down < a.rows) to[down * static_cast<int64_t>(a.w.outputs)] = total[r][c][i] * Meets<T>::kBack;
                }
            continue;
        }
        const float bias = bias_of<T>(a.bias, a.wide_bias, n);
        T* const to = a.y + m * a.y_stride + n;
#pragma unroll
        for (int r = 0; r < kB; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int down = 32 * r + 8 * (i / 4) + i % 4;
                if (m + down < a.rows) to[down * a.y_stride] = static_cast<T>(fmaf(total[r][c][i], Meets<T>::kBack, bias));
            }
    }
}

// Which kernel serves.  What counts is the units of 16 rows, 16 outputs and a span; measured on one MI355X, us, bfloat16 with groups of 128 where nothing is said:
//   kFew         small matrices: up to 8192 units, 4096 of groups of 32 (one row of 4096 x 4096 5.2, tiles of 32 rows 8.2; 16 rows 7.6 and 10.1; groups of 32, 64 rows of
//                2048 x 2048 10.7 and 8.5, 16 of 2048 x 8000 11.1 and 10.7, one 8.3 and 8.5), unless a wavefront had more than two spans (16 rows of 8192 x 2048 12.9 and 9.3).
//                Beyond both borders it is the other way from eight rows on (4096 x 6144 11.2 and 10.1, 5120 x 5120 13.1 and 10.6, 14336 x 4096 16.7 and 13.9; 8192 x 4096
//                10.7 and 11.2); one row alone would still gain (8.7 and 9.7, 9.9 and 10.2, 12.3 and 13.5, 8.3 and 10.5)
//   kFewWide     a few rows of many outputs: x is read once for 64 outputs (one row of 8192 x 16384 19.4, tiles 23.0; of 2048 x 16384 7.2 and 10.1, 16 8.7 and 11.7; binary32 10.4
//                and 18.2, 12.4 and 20.3; groups of 32 44 and 30)
//   kLowTiles    up to 64 rows, or 131072 units (binary32, where products are three times as many, 32768): 128 rows of 4096 x 4096 16.9, tiles of 128 rows 26.6;
//                192 23.1 and 26.4; 301 33.3 and 31.1; 128 of 8192 x 8192 39.7 and 35.6; binary32, 301 rows of 1000 x 1501 18.8 and 26.1, 300 of 2048 x 2048 29.7 and 27.8
//   kHighTiles   else
enum Kernel { kFew, kFewWide, kLowTiles, kHighTiles };

Kernel kernel_of(const actq_weights4* w, int dtype, int64_t rows)
{
    const int64_t spans = (w->inputs + kSpan - 1) / kSpan, units = (rows + 15) / 16 * ((w->outputs + 15) / 16) * spans;
    if (rows <= 16 && w->outputs >= 8192 && w->group >= 64) return kFewWide;
    if (spans <= 32 && units <= (w->group == 32 ? 4096 : 8192)) return kFew;
    return rows <= 64 || units <= (dtype == ACTQ_F32 ? 32768 : 131072) ? kLowTiles : kHighTiles;
}

// Whether rows of x can be taken as they lie.
bool as_they_lie(const actq_weights4* w, int dtype, const actq_rows* x)
{
    return dtype != ACTQ_F32 && w->inputs % kSpan == 0 && x->stride % 8 == 0 && reinterpret_cast<uintptr_t>(x->data) % 16 == 0;
}

int32_t padded_inputs(const actq_weights4* w) { return (w->inputs + kSpan - 1) / kSpan * kSpan; }

// The sums, then the copy of x.
uint64_t sums_bytes(const actq_weights4* w, int64_t rows) { return (static_cast<uint64_t>(rows) * (padded_inputs(w) / w->group) * sizeof(u32x2) + 15) / 16 * 16; }
uint64_t copy_bytes(const actq_weights4* w, int dtype, int64_t rows) { return static_cast<uint64_t>(rows) * padded_inputs(w) * (dtype == ACTQ_F32 ? 6 : 2); }

// Parts of the inputs: where the tiles are fewer than the compute units, as many as make one workgroup for each, of two spans at
// least (of 32 rows two for each: 32 rows of 8192 x 16384 25.8 -> 31.0 us, four 38.7).
struct Parts {
    int32_t row_tiles, column_tiles, count, share;
};

Parts parts_of(const actq_weights4* w, int64_t rows, bool low)
{
    Parts p;
    p.row_tiles = static_cast<int32_t>(low ? (rows + 31) / 32 : (rows + 127) / 128);
    p.column_tiles = (w->outputs + 255) / 256;
    const int64_t tiles = static_cast<int64_t>(p.row_tiles) * p.column_tiles, spans = padded_inputs(w) / kSpan;
    const int64_t wanted = 256 / tiles, most = wanted < spans / 2 ? wanted : spans / 2, share = most > 1 ? (spans + most - 1) / most : spans;
    p.share = static_cast<int32_t>(share * kSpan);
    p.count = static_cast<int32_t>((spans + share - 1) / share);
    return p;
}

uint64_t parts_bytes(const actq_weights4* w, int64_t rows, bool low)
{
    const Parts p = parts_of(w, rows, low);
    return p.count > 1 ? static_cast<uint64_t>(p.count) * rows * w->outputs * sizeof(float) : 0;
}

template <typename T, int GROUP>
int launch_tiles(const actq_weights4* w, const actq_rows* x, int64_t rows, bool low, const void* bias, int bias_dtype, const actq_rows* y, void* workspace, hipStream_t stream)
{
    const int dtype = sizeof(T) == 4 ? ACTQ_F32 : ACTQ_F16;
    const bool copied = !as_they_lie(w, dtype, x);
    const int32_t padded = padded_inputs(w);
    u32x2* const sums = static_cast<u32x2*>(workspace);
    u32x4* const copy = copied ? reinterpret_cast<u32x4*>(static_cast<char*>(workspace) + sums_bytes(w, rows)) : nullptr;
    PrepareArgs<T> p = {};
    p.x = static_cast<const T*>(x->data);
    p.stride = x->stride;
    p.inputs = w->inputs;
    p.padded = padded;
    p.rows = rows;
    p.copy = copy;
    p.sums = sums;
    if (!low || copied)
        launches((rows * (padded / 8) + 255) / 256, 256, [&](int64_t first, unsigned count) {
            p.first = first;
            launch(linear4_prepare_kernel<T, GROUP>, count, 256, stream, p);
        });
    ManyArgs<T> a = {};
    a.w = weights_of(w);
    a.x = copied ? reinterpret_cast<const uint16_t*>(copy) : static_cast<const uint16_t*>(x->data);
    a.x_stride = copied ? padded : x->stride;
    a.x_piece = rows * padded;
    a.sums = sums;
    a.padded = padded;
    a.bias = bias;
    a.wide_bias = bias_dtype == ACTQ_F32;
    a.y = static_cast<T*>(y->data);
    a.y_stride = y->stride;
    a.rows = rows;
    const Parts parts = parts_of(w, rows, low);
    a.row_tiles = parts.row_tiles;
    a.column_tiles = parts.column_tiles;
    a.share = parts.share;
    if (parts.count > 1) a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + sums_bytes(w, rows) + copy_bytes(w, dtype, rows));
    launch(low ? linear4_many_kernel<T, GROUP, 32> : linear4_many_kernel<T, GROUP, 128>, dim3(static_cast<unsigned>((a.row_tiles * a.column_tiles + 7) / 8 * 8), static_cast<unsigned>(parts.count)), 512, stream, a);
    if (parts.count > 1)
        launch(linear4_join_kernel<T>, static_cast<unsigned>((rows * w->outputs + 255) / 256), 256, stream, static_cast<const float*>(a.parts), parts.count, rows, w->outputs, bias,
               a.wide_bias, a.y, a.y_stride);
    return launched("actq_linear4");
}

// ----------------------------------------------------------------------------- the gradient

// Few rows.  A workgroup's tile is 128 x 128 of grad_x, gathered over 64 outputs at a time from the LDS.  A weight goes there as two bfloat16 numbers (16 bits of
// it; three for binary32), an element of grad_y as those that make it up (binary16: two, binary32: three): products below 2^-16 (2^-24) of the largest are left out.
// What bounds it: the trips to memory of its stages, one behind the other: a stage's words, headers and rows are asked for when the last one has been multiplied.  Of 31 us for one row
// of 4096 inputs and 8192 outputs (one part of the outputs: 315) turning the weights into numbers, 6 instructions a code, is some 5, the products of a tile, as many for a row
// as for 128, some 7; 64 rows 38, 128 45 (binary16 39, 46, 52; binary32 75, 84, 95).
template <typename T>
struct GradArgs {
    Weights4 w;
    const T* grad;
    int64_t grad_stride;
    T* out;
    int64_t out_stride;
    int64_t rows;
    int32_t share;   // outputs of a part
    float* parts;    // [parts][rows][inputs]; null: the only part writes out
};

template <typename T>
constexpr int kGradPieces = sizeof(T) == 4 ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;   // of an element of grad_y
template <typename T>
constexpr int kWeightPieces = sizeof(T) == 4 ? 3 : 2;

constexpr int kGradRows = 128, kGradColumns = 128, kGradDepth = 64;
constexpr int kGradThreads = 256;

// A row of the LDS is 128 bytes, eight chunks of 16, which lie at places that differ for neighbouring rows and for rows 8 apart: both kinds are accessed at once.
__device__ __forceinline__ int chunk_place(int row, int chunk) { return row * 8 + (chunk ^ ((row ^ row >> 3) & 7)); }

template <typename T, int GROUP>
__global__ __launch_bounds__(kGradThreads) void linear4_backward_kernel(GradArgs<T> a)
{
    constexpr int kGP = kGradPieces<T>, kWP = kWeightPieces<T>, kHighest = kWP > kGP ? kWP - 1 : kGP - 1;
    __shared__ u32x4 grads[kGP][kGradRows * 8];
    __shared__ u32x4 weights[kWP][kGradColumns * 8];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t first_row = static_cast<int64_t>(blockIdx.y) * kGradRows;
    const int first_column = blockIdx.x * kGradColumns, row_words = a.w.groups * (GROUP / 8);
    const int word = min(first_column / 8 + static_cast<int>(threadIdx.x % 16), row_words - 1), group = word / (GROUP / 8), quad = threadIdx.x / 16;
    f32x16 sum[2][2] = {};
    const int end = min(static_cast<int>(blockIdx.z + 1) * a.share, a.w.outputs);
    for (int from = blockIdx.z * a.share; from < end; from += kGradDepth) {
        // grad_y: chunks of eight outputs
        for (int i = threadIdx.x; i < kGradRows * 8; i += kGradThreads) {
            const int row = i / 8, chunk = i % 8, n = from + 8 * chunk;
            const int64_t m = first_row + row;
            const T* const g = a.grad + (m < a.rows ? m : a.rows - 1) * a.grad_stride;
            Eight<T> e;
            if (n + kLaneValues <= a.w.outputs) {
                e.load(g + n);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) e.v[j] = n + j < a.w.outputs ? g[n + j] : static_cast<T>(0.0f);
            }
            if constexpr (kGP == 1) {
                grads[0][chunk_place(row, chunk)] = __builtin_bit_cast(u32x4, e.v);
            } else {
                u32x4 p[kGP];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t low[kGP], high[kGP];
                    split(static_cast<float>(e.v[2 * j]), low);
                    split(static_cast<float>(e.v[2 * j + 1]), high);
#pragma unroll
                    for (int k = 0; k < kGP; ++k) p[k][j] = low[k] >> 16 | high[k];
                }
#pragma unroll
                for (int k = 0; k < kGP; ++k) grads[k][chunk_place(row, chunk)] = p[k];
            }
        }
        // weights: a word of four outputs, turned so that the outputs are neighbours
        {
            float v[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = from + 4 * quad + j;
                const bool there = n < a.w.outputs;
                const int64_t row = there ? n : 0;
                const uint32_t w = there ? a.w.codes[row * row_words + word] : 0u, h = there ? a.w.header[row * a.w.groups + group] : 0u;
                const float zero = zero_of(h), step = step_of(h);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] = fmaf(static_cast<float>(w >> (4 * (i / 2) + 16 * (i % 2)) & 15u), step, zero);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t bits[4][kWP];
#pragma unroll
                for (int j = 0; j < 4; ++j) split(v[j][i], bits[j]);
                const int row = 8 * (threadIdx.x % 16) + i, place = chunk_place(row, quad / 2);
#pragma unroll
                for (int k = 0; k < kWP; ++k)
                    reinterpret_cast<u32x2*>(&weights[k][place])[quad % 2] = u32x2{bits[0][k] >> 16 | bits[1][k], bits[2][k] >> 16 | bits[3][k]};
            }
        }
        __syncthreads();
#pragma unroll
        for (int deep = 0; deep < kGradDepth / 16; ++deep) {
            const int chunk = 2 * deep + lane / 32;
            bf16x8 g[2][kGP], w[2][kWP];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int k = 0; k < kGP; ++k) g[t][k] = __builtin_bit_cast(bf16x8, grads[k][chunk_place(64 * (wave / 2) + 32 * t + lane % 32, chunk)]);
#pragma unroll
                for (int k = 0; k < kWP; ++k) w[t][k] = __builtin_bit_cast(bf16x8, weights[k][chunk_place(64 * (wave % 2) + 32 * t + lane % 32, chunk)]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int p = kGP - 1; p >= 0; --p)
#pragma unroll
                        for (int q = kWP - 1; q >= 0; --q)
                            if (p + q <= kHighest) sum[i][j] = multiply(g[i][p], w[j][q], sum[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int k = first_column + 64 * (wave % 2) + 32 * j + lane % 32;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t m = first_row + 64 * (wave / 2) + 32 * i + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
                if (m >= a.rows || k >= a.w.inputs) continue;
                if (a.parts)
                    a.parts[(blockIdx.z * a.rows + m) * a.w.inputs + k] = sum[i][j][r];
                else
                    a.out[m * a.out_stride + k] = static_cast<T>(sum[i][j][r]);
            }
        }
}

// Many rows: the weights are turned into numbers once, transposed, in memory, and the product is one of two matrices whose rows are contiguous along the outputs.
// Both are binary16, scaled by powers of two so that it has the range: a weight by that of its output's largest one, which the elements of grad_y there make up for;
// a row of grad_y by that of its largest element, for which the row of the result makes up.  A weight is step (code - 8), which has the 11 bits of one number (8 of a step, 3 of
// up to 8), and its group's zero + 8 step, of which there is one for `group` columns: two numbers (22 bits), and a product of their own.  An element of grad_y is one number, of
// binary32 two, without the product of the second ones.
template <typename T>
constexpr int kGradNumbers = sizeof(T) == 4 ? 2 : 1;
constexpr int kMiddleNumbers = 2;

constexpr int kDeepest = 64;   // outputs are padded to a multiple

// The exponent of the power of two that takes a number of this magnitude into [2^13, 2^14): from -114 to 140.  Zero counts as
// the smallest: an output without weights, whose element of grad_y adds nothing, must not
// be its row's largest.
__device__ __forceinline__ int power_of(uint32_t largest) { return largest >= 0x7f800000u ? 0 : 140 - static_cast<int>(largest >> 23); }

__device__ __forceinline__ float two_to(int power) { return __builtin_bit_cast(float, static_cast<uint32_t>(power + 127) << 23); }   // from -126 to 127

// 1 / the scale of every output, a wavefront each: both are normal numbers, which leaves weights below 2^-113 in [0, 2^13).
__global__ __launch_bounds__(256) void weights4_scale_kernel(Weights4 w, float* inverse)
{
    const int n = blockIdx.x * 4 + threadIdx.x / 64;
    if (n >= w.outputs) return;
    uint32_t largest = 0;
    for (int g = threadIdx.x % 64; g < w.groups; g += 64) {
        const uint32_t h = w.header[static_cast<int64_t>(n) * w.groups + g];
        const uint32_t ends[2] = {magnitude(zero_of(h)), magnitude(fmaf(15.0f, step_of(h), zero_of(h)))};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (ends[i] < 0x7f800000u) largest = max(largest, ends[i]);
    }
#pragma unroll
    for (int step = 1; step < 64; step *= 2) largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), step)));
    if (threadIdx.x % 64 == 0) inverse[n] = two_to(-min(power_of(largest), 126));
}

// 64 outputs x 128 inputs a workgroup; out [inputs][padded outputs], middles [groups][numbers][padded outputs].
template <int GROUP>
__global__ __launch_bounds__(256) void weights4_transpose_kernel(Weights4 w, const float* inverse, int32_t padded, uint16_t* out, uint16_t* middles)
{
    typedef _Float16 four __attribute__((ext_vector_type(4)));
    __shared__ u32x2 turned[128 * 17];
    const int row_words = w.groups * (GROUP / 8), column = threadIdx.x % 16, quad = threadIdx.x / 16, wanted = blockIdx.x * 16 + column;
    const int word = min(wanted, row_words - 1), group = word / (GROUP / 8);
    float v[4][8], middle[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = blockIdx.y * 64 + 4 * quad + j;
        const bool there = n < w.outputs;
        const int64_t row = there ? n : 0;
        const uint32_t codes = w.codes[row * row_words + word], h = there ? w.header[row * w.groups + group] : 0u;
        const float scale = 1.0f / inverse[row], step = step_of(h) * scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = (static_cast<float>(codes >> (4 * (i / 2) + 16 * (i % 2)) & 15u) - 8.0f) * step;
        middle[j] = fmaf(8.0f, step_of(h), zero_of(h)) * scale;
    }
    if (wanted < row_words && column % (GROUP / 8) == 0) {
#pragma unroll
        for (int number = 0; number < kMiddleNumbers; ++number) {
            four f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[j] = static_cast<_Float16>(middle[j]);
                middle[j] -= static_cast<float>(f[j]);
            }
            *reinterpret_cast<four*>(middles + (static_cast<int64_t>(group) * kMiddleNumbers + number) * padded + blockIdx.y * 64 + 4 * quad) = f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        four f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = static_cast<_Float16>(v[j][i]);
        turned[(8 * column + i) * 17 + quad] = __builtin_bit_cast(u32x2, f);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 32 + threadIdx.x / 8, pair = threadIdx.x % 8 * 2, k = blockIdx.x * 128 + row;
        const u32x2 a = turned[row * 17 + pair], b = turned[row * 17 + pair + 1];
        if (k < w.inputs) *reinterpret_cast<u32x4*>(out + static_cast<int64_t>(k) * padded + blockIdx.y * 64 + 4 * pair) = u32x4{a[0], a[1], b[0], b[1]};
    }
}

// A row of grad_y a workgroup; out [numbers][rows][padded outputs], and what its result has to be multiplied by.
template <typename T>
__global__ __launch_bounds__(256) void linear4_scale_rows_kernel(const T* grad, int64_t stride, int64_t rows, int32_t outputs, int32_t padded, const float* inverse, uint16_t* out, float* back)
{
    __shared__ uint32_t shares[4];
    const int64_t m = blockIdx.x;
    const T* const row = grad + m * stride;
    const auto at = [&](int n, float (&f)[8]) {
        Eight<T> e;
        Eight<float> by;
        if (n + 8 <= outputs) {
            e.load(row + n);
            by.load(inverse + n);
            e.widen(f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= by.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = n + i < outputs ? static_cast<float>(row[n + i]) * inverse[n + i] : 0.0f;
        }
    };
    uint32_t largest = 0;
    for (int n = 8 * threadIdx.x; n < outputs; n += 8 * 256) {
        float f[8];
        at(n, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(f[i]));
    }
#pragma unroll
    for (int step = 1; step < 64; step *= 2) largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), step)));
    if (threadIdx.x % 64 == 0) shares[threadIdx.x / 64] = largest;
    __syncthreads();
    largest = max(max(shares[0], shares[1]), max(shares[2], shares[3]));
    // in two steps, as one of them has no room for the smallest numbers
    const int power = power_of(largest), half = power / 2;
    const float first = two_to(half), second = two_to(power - half);
    if (threadIdx.x == 0) back[m] = two_to(-half) * two_to(half - power);
    for (int n = 8 * threadIdx.x; n < padded; n += 8 * 256) {
        float f[8];
        at(n, f);
#pragma unroll
        for (int number = 0; number < kGradNumbers<T>; ++number) {
            f16x8 v;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (number == 0) f[i] = f[i] * first * second;
                v[i] = static_cast<_Float16>(f[i]);
                f[i] -= static_cast<float>(v[i]);
            }
            *reinterpret_cast<u32x4*>(out + (static_cast<int64_t>(number) * rows + m) * padded + n) = __builtin_bit_cast(u32x4, v);
        }
    }
}

template <typename T>
struct TilesArgs {
    const uint16_t* grad;     // [numbers][rows][padded]
    const uint16_t* weights;  // [inputs][padded]; of the middles [groups][numbers][padded], all of which are inputs here
    const float* back;
    const float* middles;     // [groups][padded_rows], what comes to a row's sums in a group
    int32_t group_shift;
    int64_t rows, padded_rows;   // whole tiles
    int32_t inputs, padded;
    int32_t row_tiles, column_tiles;
    T* out;
    int64_t out_stride;
    int32_t share;            // outputs of a part
    float* parts;             // [parts][rows][inputs]; null: the only part writes out.  Of the middles [parts][groups][padded_rows], and nothing else
};

// A workgroup's tile is 256 rows x 128 inputs, a wavefront's 128 x 64, and both matrices go from memory to the LDS without registers, two stages ahead.
// What bounds it: the matrix instructions, beside which the LDS is read three quarters of the time.
template <typename T, int GRADS, bool MIDDLES>
__global__ __launch_bounds__(256, 1) void linear4_backward_tiles_kernel(TilesArgs<T> a)
{
    constexpr int kG = GRADS, kDepth = kG == 1 ? 64 : 32, kRing = 3, kRows = 256, kColumns = 128;
    constexpr int kChunks = kDepth / 8, kGrads = kRows * kChunks, kWeights = kColumns * kChunks, kStage = kG * kGrads + kWeights, kLoads = kStage / 256;
    __shared__ u32x4 lds[kRing * kStage];   // one array, as above
    const int lane = threadIdx.x % 64, at = lane % 32, half = lane / 32;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), rows = wave / 2 * 128, columns = wave % 2 * 64;
    const int tiles = a.row_tiles * a.column_tiles, share = (tiles + 7) / 8, unit = blockIdx.x % 8 * share + blockIdx.x / 8;
    if (unit >= tiles || static_cast<int>(blockIdx.x / 8) >= share) return;
    const int band = unit / (4 * a.column_tiles), in_band = unit - band * 4 * a.column_tiles, high = min(4, a.row_tiles - 4 * band);
    const int64_t first_row = static_cast<int64_t>(4 * band + in_band % high) * kRows;
    const int first_column = (in_band / high) * kColumns;
    const auto swizzle = [](int row) { return kChunks == 8 ? row & 7 : row >> 2 & 3; };
    const uint16_t* from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const bool of_grad = i * 256 < kG * kGrads;
        const int place = i * 256 + threadIdx.x - (of_grad ? 0 : kG * kGrads), number = place / (of_grad ? kGrads : kWeights), in = place % (of_grad ? kGrads : kWeights);
        const int row = in / kChunks, chunk = in % kChunks ^ swizzle(row);
        const int64_t all = of_grad ? a.rows : a.inputs, wanted = (of_grad ? first_row : first_column) + row;
        from[i] = (of_grad ? a.grad : a.weights) + (number * all + (wanted < all ? wanted : all - 1)) * a.padded + 8 * chunk;
    }
    const auto load = [&](int n, int to) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) to_lds(from[i] + n, lds + to * kStage + i * 256 + wave * 64);
    };
    const int begin = blockIdx.y * a.share, end = min(begin + a.share, a.padded);
    load(begin, 0);
    if (begin + kDepth < end) load(begin + kDepth, 1);
    f32x16 sum[4][2] = {};
    if (begin + kDepth < end)
        arrived<kLoads>();
    else
        arrived<0>();
    int buffer = 0;
    for (int n = begin; n < end; n += kDepth) {
        const int ahead = n + (kRing - 1) * kDepth;
        if (ahead < end) load(ahead, buffer == 0 ? kRing - 1 : buffer - 1);
        const u32x4* const stage = lds + buffer * kStage;
#pragma unroll
        for (int step = 0; step < kDepth / 16; ++step) {
            f16x8 g[4][kG], w[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = rows + 32 * i + at;
#pragma unroll
                for (int p = 0; p < kG; ++p) g[i][p] = __builtin_bit_cast(f16x8, stage[p * kGrads + row * kChunks + ((2 * step + half) ^ swizzle(row))]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = columns + 32 * j + at;
                w[j] = __builtin_bit_cast(f16x8, stage[kG * kGrads + row * kChunks + ((2 * step + half) ^ swizzle(row))]);
            }
#pragma unroll
            for (int p = kG - 1; p >= 0; --p)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) sum[i][j] = multiply(g[i][p], w[j], sum[i][j]);
        }
        if (ahead < end)
            arrived<(kRing - 2) * kLoads>();
        else
            arrived<0>();
        buffer = buffer == kRing - 1 ? 0 : buffer + 1;
    }
    // four neighbouring rows a lane and register quad; what goes with them is loaded for 32 rows at a time (one by one: 22 us more)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t first = first_row + rows + 32 * i + 4 * half;
        if constexpr (MIDDLES) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int k = first_column + columns + 32 * j + at;
                    f32x4 v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = sum[i][j][4 * q + r] + dpp<kDppXor1>(sum[i][j][4 * q + r]);   // of both numbers
                    if (k < a.inputs && k % kMiddleNumbers == 0)
                        *reinterpret_cast<f32x4*>(a.parts + ((static_cast<int64_t>(blockIdx.y) * a.inputs + k) / kMiddleNumbers) * a.padded_rows + first + 8 * q) = v;
                }
        } else {
            f32x4 back[4], middle[2][4] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                back[q] = *reinterpret_cast<const f32x4*>(a.back + first + 8 * q);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int64_t group = min(first_column + columns + 32 * j, a.inputs - 1) >> a.group_shift;
                    if (blockIdx.y == 0) middle[j][q] = *reinterpret_cast<const f32x4*>(a.middles + group * a.padded_rows + first + 8 * q);
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t m = first + 8 * (r / 4) + r % 4;
                if (m >= a.rows) continue;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int k = first_column + columns + 32 * j + at;
                    if (k >= a.inputs) continue;
                    const float v = (sum[i][j][r] + middle[j][r / 4][r % 4]) * back[r / 4][r % 4];
                    if (a.parts)
                        a.parts[(blockIdx.y * a.rows + m) * a.inputs + k] = v;
                    else
                        a.out[m * a.out_stride + k] = static_cast<T>(v);
                }
            }
        }
    }
}

// ----------------------------------------------------------------------------- the bias

// Sums of columns.  A wavefront takes every fourth row of its workgroup's, 512 columns of it, four rows in flight, whose sums are binary32 and above them binary64; the workgroups' sums are
// added up by a second kernel.  What bounds it: memory (a library's sum of many rows clears its counters with an operation of its own, which graphs
// do not replay rightly here).
constexpr int kBiasColumns = 512, kBiasAhead = 4;

template <typename T>
__global__ __launch_bounds__(256) void linear4_bias_kernel(const T* grad, int64_t stride, int64_t rows, int64_t share, int32_t outputs, float* parts, void* out, int wide)
{
    __shared__ double sums[4][kBiasColumns];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), column = blockIdx.x * kBiasColumns + kLaneValues * lane;
    const int64_t begin = blockIdx.y * share, end = begin + share < rows ? begin + share : rows;
    double sum[8] = {};
    for (int64_t m = begin + wave; m < end; m += 4 * kBiasAhead) {
        Eight<T> e[kBiasAhead];
#pragma unroll
        for (int u = 0; u < kBiasAhead; ++u) {
            const T* const row = grad + (m + 4 * u) * stride;
            e[u].v = {};
            if (m + 4 * u < end && column + kLaneValues <= outputs) {
                e[u].load(row + column);
            } else if (m + 4 * u < end) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (column + i < outputs) e[u].v[i] = row[column + i];
            }
        }
        float four[8] = {};
#pragma unroll
        for (int u = 0; u < kBiasAhead; ++u) {
            float f[8];
            e[u].widen(f);
#pragma unroll
            for (int i = 0; i < 8; ++i) four[i] += f[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += static_cast<double>(four[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][kLaneValues * lane + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < kBiasColumns; i += 256) {
        const int n = blockIdx.x * kBiasColumns + i;
        if (n >= outputs) continue;
        const float all = static_cast<float>((sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]));
        if (parts)
            parts[static_cast<int64_t>(blockIdx.y) * outputs + n] = all;
        else if (wide)
            static_cast<float*>(out)[n] = all;
        else
            static_cast<T*>(out)[n] = static_cast<T>(all);
    }
}

// 16 columns a workgroup, 16 threads for each.
template <typename W>
__global__ __launch_bounds__(256) void linear4_bias_join_kernel(const float* parts, int32_t count, int32_t outputs, W* out)
{
    __shared__ double sums[16][16];
    const int at = threadIdx.x % 16, row = threadIdx.x / 16, n = blockIdx.x * 16 + at;
    double sum = 0.0;
#pragma unroll 4
    for (int i = row; i < count; i += 16) sum += n < outputs ? static_cast<double>(parts[static_cast<int64_t>(i) * outputs + n]) : 0.0;
    sums[row][at] = sum;
    __syncthreads();
    if (row > 0 || n >= outputs) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += sums[i][at];
    out[n] = static_cast<W>(static_cast<float>(sum));
}

// Parts of the rows: two workgroups a compute unit, of 16 rows at least.
int32_t bias_parts(int64_t rows, int32_t outputs)
{
    const int64_t tiles = (outputs + kBiasColumns - 1) / kBiasColumns, most = (rows + 15) / 16, wanted = 512 / tiles < most ? 512 / tiles : most;
    return static_cast<int32_t>(wanted > 1 ? wanted : 1);
}

// ----------------------------------------------------------------------------- the weights themselves

// A thread is a word.  zero = min and step = (max - min) / 15 are rounded to bfloat16 before the codes are worked out with them; a group with an infinity or
// NaN, or whose zero or step overflows, reads as NaN.
template <typename T>
__global__ __launch_bounds__(256) void weights4_quantize_kernel(const T* w, int64_t stride, int32_t inputs, int32_t group, int32_t row_words, int64_t words, int64_t first, uint32_t* codes, uint32_t* header)
{
    const int64_t unit = (first + blockIdx.x) * 256 + threadIdx.x;
    const bool there = unit < words;
    const int64_t n = there ? unit / row_words : 0;
    const int word = there ? static_cast<int>(unit - n * row_words) : 0;
    const T* const row = w + n * stride;
    float x[8], low = INFINITY, high = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = 8 * word + i;
        x[i] = 0.0f;
        if (k < inputs) x[i] = static_cast<float>(row[k]);
        if (magnitude(x[i]) >= 0x7f800000u) {
            bad = true;
            x[i] = 0.0f;
        }
        if (k < inputs) {
            low = fminf(low, x[i]);
            high = fmaxf(high, x[i]);
        }
    }
    int none = bad;
    for (int step = 1; step < group / 8; step *= 2) {
        low = fminf(low, __shfl_xor(low, step));
        high = fmaxf(high, __shfl_xor(high, step));
        none |= __shfl_xor(none, step);
    }
    const float zero = static_cast<float>(static_cast<__bf16>(low + 0.0f));
    float step = static_cast<float>(static_cast<__bf16>((high - low) / 15.0f));
    none = none || magnitude(zero) >= 0x7f800000u || magnitude(step) >= 0x7f800000u;
    float inverse = 1.0f / step;
    if (step == 0.0f || isinf(inverse)) inverse = step = 0.0f;
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float code = none || 8 * word + i >= inputs ? 0.0f : rintf(fminf(fmaxf((x[i] - zero) * inverse, 0.0f), 15.0f));
        out |= static_cast<uint32_t>(code) << (4 * (i / 2) + 16 * (i % 2));
    }
    if (!there) return;
    codes[unit] = out;
    if (word % (group / 8) == 0)
        header[n * (row_words / (group / 8)) + word / (group / 8)] = none ? 0x7fc07fc0u : __builtin_bit_cast(uint32_t, zero) >> 16 | __builtin_bit_cast(uint32_t, step);
}

template <typename T>
__global__ __launch_bounds__(256) void weights4_dequantize_kernel(Weights4 w, int32_t group, int64_t words, int64_t first, T* out, int64_t stride)
{
    const int64_t unit = (first + blockIdx.x) * 256 + threadIdx.x;
    if (unit >= words) return;
    const int row_words = w.groups * (group / 8);
    const int64_t n = unit / row_words;
    const int word = static_cast<int>(unit - n * row_words);
    const uint32_t code = w.codes[unit], h = w.header[n * w.groups + word / (group / 8)];
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = static_cast<T>(fmaf(static_cast<float>(code >> (4 * (i / 2) + 16 * (i % 2)) & 15u), step_of(h), zero_of(h)));
    T* const to = out + n * stride + 8 * word;
    if (8 * word + 8 <= w.inputs) {
        e.store(to);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (8 * word + i < w.inputs) to[i] = e.v[i];
    }
}

template <typename F>
int by_group(int32_t group, F f)
{
    return group == 32 ? f(std::integral_constant<int, 32>{}) : group == 64 ? f(std::integral_constant<int, 64>{}) : f(std::integral_constant<int, 128>{});
}

}  // namespace

int launch_weights4_quantize(const actq_rows* w, int dtype, const actq_weights4* to, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        typedef decltype(type) T;
        const Weights4 v = weights_of(to);
        const int32_t row_words = v.groups * (to->group / 8);
        const int64_t words = static_cast<int64_t>(v.outputs) * row_words;
        launches((words + 255) / 256, 256, [&](int64_t first, unsigned count) {
            launch(weights4_quantize_kernel<T>, count, 256, static_cast<hipStream_t>(stream), static_cast<const T*>(w->data), w->stride, to->inputs, to->group, row_words, words, first,
                   const_cast<uint32_t*>(v.codes), const_cast<uint32_t*>(v.header));
        });
        return launched("actq_weights4_quantize");
    });
}

int launch_weights4_dequantize(const actq_weights4* w, const actq_rows* out, int dtype, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        typedef decltype(type) T;
        const Weights4 v = weights_of(w);
        const int64_t words = static_cast<int64_t>(v.outputs) * v.groups * (w->group / 8);
        launches((words + 255) / 256, 256, [&](int64_t first, unsigned count) {
            launch(weights4_dequantize_kernel<T>, count, 256, static_cast<hipStream_t>(stream), v, w->group, words, first, static_cast<T*>(out->data), out->stride);
        });
        return launched("actq_weights4_dequantize");
    });
}

uint64_t linear4_workspace(const actq_weights4* w, int dtype, int64_t rows)
{
    if (rows == 0) return 0;
    const Kernel kernel = kernel_of(w, dtype, rows);
    return kernel == kFew || kernel == kFewWide ? 0 : sums_bytes(w, rows) + copy_bytes(w, dtype, rows) + parts_bytes(w, rows, kernel == kLowTiles);
}

// Whether the weights are turned into numbers in memory, two bytes for each: from so many products on, and so many rows, which make up for writing them.  The other kernel
// takes a tile of 128 rows in little more time than one.  us, from memory and by the other kernel, groups of 128:
//   bfloat16  256 rows, 4096 inputs, 8192 outputs 83, 71; 384 99, 104; 8192 rows of 1024 x 1024 67, 64; 1500 of 2048 x 2048 66, 71; 128 rows of 8192 x 65536 784, 536; 129 789, 998
//   binary16  192 rows, 4096 inputs, 8192 outputs 80, 83; 1024 of 2048 x 2048 58, 53; 1500 67, 86; 128 of 8192 x 65536 787, 648; 129 789, 1237
//   binary32  512 rows of 2048 x 2048 59, 61; 1024 70, 99; 128 rows, 4096 inputs, 8192 outputs 95, 95; 64 of 8192 x 16384 271, 291; 64 of 8192 x 65536 990, 1257, for which it takes
//             no GiB; 100 1014, 1406
bool in_memory(const actq_weights4* w, int dtype, int64_t rows)
{
    return rows > (dtype == ACTQ_F32 ? 64 : 128) && rows * w->inputs * w->outputs > int64_t(1) << (dtype == ACTQ_F32 ? 31 : dtype == ACTQ_F16 ? 32 : 33);
}

struct GradPlan {
    bool tiles;               // of 256 rows, from numbers in memory
    int32_t row_tiles, column_tiles, padded, share, parts;
    int32_t middle_share, middle_parts;
    uint64_t inverse, back, grads, weights, middles, middle_sums, sums;   // bytes of the workspace's pieces
};

// Outputs of a part (a multiple of kDeepest) and how many parts: as many as make `wanted` of the tiles, of `least` stages at least.
void cut_outputs(int32_t padded, int64_t tiles, int64_t wanted, int64_t least, int32_t& share, int32_t& parts)
{
    const int64_t stages = padded / kDeepest, most = wanted / tiles < stages / least ? wanted / tiles : stages / least, each = most > 1 ? (stages + most - 1) / most : stages;
    share = static_cast<int32_t>(each * kDeepest);
    parts = static_cast<int32_t>((stages + each - 1) / each);
}

// Where the tiles are few, the outputs are cut into parts that make a workgroup for each compute unit (of the smaller tiles two), of four stages at least.
GradPlan grad_plan(const actq_weights4* w, int dtype, int64_t rows)
{
    GradPlan p = {};
    if (rows == 0) return p;
    p.tiles = in_memory(w, dtype, rows);
    p.row_tiles = static_cast<int32_t>(p.tiles ? (rows + 255) / 256 : (rows + kGradRows - 1) / kGradRows);
    p.column_tiles = (w->inputs + kGradColumns - 1) / kGradColumns;
    p.padded = (w->outputs + kDeepest - 1) / kDeepest * kDeepest;
    cut_outputs(p.padded, static_cast<int64_t>(p.row_tiles) * p.column_tiles, p.tiles ? 256 : 512, 4, p.share, p.parts);
    if (p.tiles) {
        const int32_t groups = (w->inputs + w->group - 1) / w->group;
        cut_outputs(p.padded, static_cast<int64_t>(p.row_tiles) * ((kMiddleNumbers * groups + kGradColumns - 1) / kGradColumns), 256, 4, p.middle_share, p.middle_parts);
        p.inverse = (static_cast<uint64_t>(w->outputs) * sizeof(float) + 15) / 16 * 16;
        const uint64_t padded_rows = static_cast<uint64_t>(p.row_tiles) * 256;
        p.back = padded_rows * sizeof(float);
        p.grads = static_cast<uint64_t>(rows) * p.padded * 2 * (dtype == ACTQ_F32 ? 2 : 1);
        p.weights = static_cast<uint64_t>(w->inputs) * p.padded * 2;
        p.middles = static_cast<uint64_t>(groups) * p.padded * 2 * kMiddleNumbers;
        p.middle_sums = padded_rows * groups * sizeof(float) * (p.middle_parts > 1 ? p.middle_parts + 1 : 1);
    }
    p.sums = p.parts > 1 ? static_cast<uint64_t>(p.parts) * rows * w->inputs * sizeof(float) : 0;
    return p;
}

uint64_t linear4_backward_workspace(const actq_weights4* w, int dtype, int64_t rows)
{
    const GradPlan p = grad_plan(w, dtype, rows);
    return p.inverse + p.back + p.grads + p.weights + p.middles + p.middle_sums + p.sums;
}

template <typename T, int GROUP>
void launch_backward_tiles(const actq_weights4* w, const actq_rows* grad_y, int64_t rows, const actq_rows* grad_x, const GradPlan& p, void* workspace, float* parts, hipStream_t stream)
{
    char* const at = static_cast<char*>(workspace);
    float* const inverse = reinterpret_cast<float*>(at);
    float* const back = reinterpret_cast<float*>(at + p.inverse);
    uint16_t* const grads = reinterpret_cast<uint16_t*>(at + p.inverse + p.back);
    uint16_t* const weights = reinterpret_cast<uint16_t*>(at + p.inverse + p.back + p.grads);
    uint16_t* const middles = reinterpret_cast<uint16_t*>(at + p.inverse + p.back + p.grads + p.weights);
    float* const middle_sums = reinterpret_cast<float*>(at + p.inverse + p.back + p.grads + p.weights + p.middles);
    const Weights4 v = weights_of(w);
    launch(weights4_scale_kernel, static_cast<unsigned>((w->outputs + 3) / 4), 256, stream, v, inverse);
    launch(weights4_transpose_kernel<GROUP>, dim3(static_cast<unsigned>((w->inputs + 127) / 128), static_cast<unsigned>(p.padded / 64)), 256, stream, v,
           static_cast<const float*>(inverse), p.padded, weights, middles);
    launch(linear4_scale_rows_kernel<T>, static_cast<unsigned>(rows), 256, stream, static_cast<const T*>(grad_y->data), grad_y->stride, rows, w->outputs, p.padded,
           static_cast<const float*>(inverse), grads, back);
    const auto grid = [](int32_t row_tiles, int32_t column_tiles, int32_t count) {
        return dim3(static_cast<unsigned>((static_cast<int64_t>(row_tiles) * column_tiles + 7) / 8 * 8), static_cast<unsigned>(count));
    };
    // what the groups' middles come to; parts of it lie behind it
    const int64_t padded_rows = static_cast<int64_t>(p.row_tiles) * 256;
    TilesArgs<T> a = {};
    a.grad = grads;
    a.weights = middles;
    a.rows = rows;
    a.padded_rows = padded_rows;
    a.inputs = kMiddleNumbers * v.groups;
    a.padded = p.padded;
    a.row_tiles = p.row_tiles;
    a.column_tiles = (a.inputs + kGradColumns - 1) / kGradColumns;
    a.share = p.middle_share;
    a.parts = p.middle_parts > 1 ? middle_sums + padded_rows * v.groups : middle_sums;
    launch(linear4_backward_tiles_kernel<T, kGradNumbers<T>, true>, grid(a.row_tiles, a.column_tiles, p.middle_parts), 256, stream, a);
    if (p.middle_parts > 1)
        launch(linear4_join_kernel<float>, static_cast<unsigned>((padded_rows * v.groups + 255) / 256), 256, stream, static_cast<const float*>(a.parts), p.middle_parts, v.groups,
               static_cast<int32_t>(padded_rows), static_cast<const void*>(nullptr), 0, middle_sums, padded_rows);
    a.weights = weights;
    a.back = back;
    a.middles = middle_sums;
    a.group_shift = __builtin_ctz(GROUP);
    a.inputs = w->inputs;
    a.column_tiles = p.column_tiles;
    a.out = static_cast<T*>(grad_x->data);
    a.out_stride = grad_x->stride;
    a.share = p.share;
    a.parts = parts;
    launch(linear4_backward_tiles_kernel<T, kGradNumbers<T>, false>, grid(p.row_tiles, p.column_tiles, p.parts), 256, stream, a);
}

int launch_linear4(const actq_weights4* w, const actq_rows* x, int dtype, int64_t rows, const void* bias, int bias_dtype, const actq_rows* y, void* workspace, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        return by_group(w->group, [&](auto g) {
            typedef decltype(type) T;
            constexpr int kGroup = decltype(g)::value;
            const Kernel kernel = kernel_of(w, dtype, rows);
            if (kernel == kLowTiles || kernel == kHighTiles)
                return launch_tiles<T, kGroup>(w, x, rows, kernel == kLowTiles, bias, bias_dtype, y, workspace, static_cast<hipStream_t>(stream));
            FewArgs<T> a = {};
            a.w = weights_of(w);
            a.x = static_cast<const T*>(x->data);
            a.x_stride = x->stride;
            a.bias = bias;
            a.wide_bias = bias_dtype == ACTQ_F32;
            a.y = static_cast<T*>(y->data);
            a.y_stride = y->stride;
            a.rows = rows;
            const auto go = [&](auto columns, auto waves) {
                constexpr int kColumns = decltype(columns)::value, kWaves = decltype(waves)::value;
                const dim3 grid((a.w.outputs + 16 * kColumns - 1) / (16 * kColumns), static_cast<unsigned>((rows + 15) / 16));
                launch(linear4_few_kernel<T, kGroup, kColumns, kWaves>, grid, 64 * kWaves, static_cast<hipStream_t>(stream), a);
                return launched("actq_linear4");
            };
            if constexpr (kGroup >= 64)
                if (kernel == kFewWide) return go(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
            return go(std::integral_constant<int, 1>{}, std::integral_constant<int, 16>{});
        });
    });
}

int launch_linear4_backward(const actq_weights4* w, const actq_rows* grad_y, int dtype, int64_t rows, const actq_rows* grad_x, void* workspace, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        return by_group(w->group, [&](auto g) {
            typedef decltype(type) T;
            constexpr int kGroup = decltype(g)::value;
            const GradPlan p = grad_plan(w, dtype, rows);
            const hipStream_t at = static_cast<hipStream_t>(stream);
            float* const parts = p.parts > 1 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.inverse + p.back + p.grads + p.weights + p.middles + p.middle_sums) : nullptr;
            if (p.tiles) {
                launch_backward_tiles<T, kGroup>(w, grad_y, rows, grad_x, p, workspace, parts, at);
            } else {
                GradArgs<T> a = {};
                a.w = weights_of(w);
                a.grad = static_cast<const T*>(grad_y->data);
                a.grad_stride = grad_y->stride;
                a.out = static_cast<T*>(grad_x->data);
                a.out_stride = grad_x->stride;
                a.rows = rows;
                a.share = p.share;
                a.parts = parts;
                const dim3 grid(static_cast<unsigned>(p.column_tiles), static_cast<unsigned>(p.row_tiles), static_cast<unsigned>(p.parts));
                launch(linear4_backward_kernel<T, kGroup>, grid, kGradThreads, at, a);
            }
            if (parts)
                launch(linear4_join_kernel<T>, static_cast<unsigned>((rows * w->inputs + 255) / 256), 256, at, static_cast<const float*>(parts), p.parts, rows, w->inputs,
                       static_cast<const void*>(nullptr), 0, static_cast<T*>(grad_x->data), grad_x->stride);
            return launched("actq_linear4_backward");
        });
    });
}

uint64_t linear4_backward_bias_workspace(int64_t rows, int32_t outputs)
{
    const int32_t parts = bias_parts(rows, outputs);
    return parts > 1 ? static_cast<uint64_t>(parts) * outputs * sizeof(float) : 0;
}

int launch_linear4_backward_bias(const actq_rows* grad_y, int dtype, int64_t rows, int32_t outputs, void* grad_bias, int bias_dtype, void* workspace, void* stream)
{
    const hipStream_t at = static_cast<hipStream_t>(stream);
    const int32_t parts = bias_parts(rows, outputs);
    float* const sums = parts > 1 ? static_cast<float*>(workspace) : nullptr;
    by_dtype(dtype, [&](auto type) {
        typedef decltype(type) T;
        launch(linear4_bias_kernel<T>, dim3(static_cast<unsigned>((outputs + kBiasColumns - 1) / kBiasColumns), static_cast<unsigned>(parts)), 256, at, static_cast<const T*>(grad_y->data),
               grad_y->stride, rows, (rows + parts - 1) / parts, outputs, sums, grad_bias, static_cast<int>(bias_dtype == ACTQ_F32));
        return ACTQ_OK;
    });
    if (sums)
        by_dtype(bias_dtype, [&](auto type) {
            typedef decltype(type) W;
            launch(linear4_bias_join_kernel<W>, static_cast<unsigned>((outputs + 15) / 16), 256, at, static_cast<const float*>(sums), parts, outputs, static_cast<W*>(grad_bias));
            return ACTQ_OK;
        });
    return launched("actq_linear4_backward_bias");
}

}  // namespace actq
