// Attention of new tokens over a paged, quantised cache.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(x_j - m),  x_j = log2(e) cap(scale q . k_j)
//
// with k_j = Zk_j + step_j code_j and v_j likewise.  The codes stay whole numbers: as they are, a byte or a nibble under zeros, they
// are subnormal binary16 numbers code * 2^-24, whose products the matrix instructions round no further than in summing them, so that
//   q . k_j = step_j 2^24 (q . code_j 2^-24) + Zk_j sum(q)
// is off by that sum alone.  The terms of a sum are cut at so many bits below where the largest one could begin; a sum of 32 products of bytes is off by 2^-21
// of the largest one (2^-19 at worst), of nibbles, with their leading zeros, by 2^-20 (2^-16): a sixteenth of what rounding a binary16 result costs, for which
// moving every nibble up is too dear (32 sequences of up to 16384, 4 bits 81.5 -> 86 us).  A row of q is scaled by a power of two of its own, so that its
// largest element fills binary16's range: exact for 16-bit types but for elements below 2^-27 of the row's largest one (2^-23 beside keys of 4 bits),
// while binary32 takes two binary16 numbers, 22 bits, and centred codes, which have no leading zeros.  Scores stay in the row's unit until the exponential,
// whose subtraction of m multiplies by the unit in the same instruction.  What one row of q holds has so no part in another's; a row with an element that is no
// finite number is none.
// The values' codes are centred, u_j = code_j - c, and
//   sum_j p_j v_j = sum_j (p_j step_j) u_j + sum_j p_j (Zv_j + c step_j),
// the second sum in binary32, one number per row.  p_j step_j is rounded to binary16 (to two of them for binary32 outputs); centred codes keep
// that error at what rounding the values themselves would cost.  So that it fits, m is the row's running maximum not of x_j but of
// x_j + log2(step_j), or log2 of a 128th of the value's middle where that is more (its sum then stays in range, and the step's share of the
// result is the smaller): what a row does not see, or hardly weighs, takes no bits from what it does.
//
// Scores are computed transposed, keys by rows: a lane holds keys of one row, so that maximum and sum are per lane, and the
// probabilities are already laid out as the right operand of the second product, whose keys come in the same order.  A group's
// constants lie in the lanes of the 16-lane row that needs them and are broadcast by the instruction that uses them (DPP).
// m moves only when a row's p_j step_j would pass 2^15, and then to where it is 2^7, so that sums are rarely rescaled.  Whether it has to is asked of the
// largest score and the largest step of a block of keys; only where those two together would pass is it worked out key by key.
//
// Where there are few rows the keys are cut into parts, whose outputs a second kernel joins.
//
// Measured on one MI355X (a large library product 1.1 PFLOP/s, a copy 5.2 TB/s).  Few rows are bound by memory where all compute units
// have work and registers suffice: 64 sequences of 8192 tokens, 32 heads over 8 of 128, 8 bits 208 us, 4 bits 110 us (both 5.5 TB/s); 32 sequences of lengths up
// to 16384 (4 bits) 78 + 5 us (4.0), the longest ones' workgroups being the last; heads of 256 spill (32 sequences of 8192, 8 bits: bfloat16 318 us, 3.5 TB/s, binary32
// 557 us, 2.0; binary32 of 128 182 us, 3.1).  Many rows are bound by vector instructions (53 % of a SIMD's cycles) and products (31 %) that hardly overlap:
// 2048 tokens over 32768, 8 bits, bfloat16 1.35 ms (790 TFLOP/s).  The error against 64 bits: binary32 1e-7 to 4e-7 of the result; 16-bit types that
// of the result's own rounding, up to 3 % more.
#include "actq_heads.h"

namespace actq {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kNothing = -3.0e38f;   // running maximum of a row that has seen no key
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMostWeight = 15.0f;   // p * step stays below 2^kMostWeight, inside binary16's range,
constexpr float kNewWeight = 7.0f;     // and below 2^kNewWeight where the running maximum has just moved
constexpr int kUnitBits = 9;           // centred codes are held as code * 2^-9
constexpr float kMostCap = 0x1p60f, kLeastCap = 0x1p-60f;
constexpr int kRowBits = 13;           // a row of q is scaled to a largest element of 2^13 to 2^14 (2^15 at the upper end of binary32's range)

struct AttendArgs {
    const uint8_t* key_codes;
    const float* key_header;
    const uint8_t* value_codes;
    const float* value_header;
    int64_t pages;
    int32_t page_shift, kv_heads;
    int32_t key_bits, value_bits;
    HeadsOf<const void> q;      // strides in elements of dtype
    HeadsOf<void> out;
    int32_t dtype;
    int32_t tokens, sequences, q_heads, group;
    FastDiv by_group;
    const int32_t* table;
    int32_t table_width;
    const int32_t* lengths;
    const int32_t* query_start;
    float factor;               // scale * log2(e); with a cap scale / cap
    float cap;                  // softcap * log2(e); 0: none
    int32_t window;             // 0: none
    float least;                // log2 of the step that smaller ones count as, so that the sum of p stays inside binary32's range
    uint32_t tiles, parts;      // row tiles of the grid, parts of the keys
    FastDiv by_tiles, by_parts, by_heads;
    int32_t per_part;           // keys of a part, a multiple of the kernels' block of keys
    float* partial;             // [parts][tokens * q_heads][dim], null: one part
    f32x2* partial_sums;        // [parts][tokens * q_heads]: running maximum and sum; no sum: nothing in sight, and no outputs written
};

__device__ __forceinline__ uint32_t divide(uint32_t n, FastDiv by) { return (__umulhi(n, by.m) + n) >> by.s; }

// What a workgroup is for.
struct Work {
    int32_t sequence, head, part, tile;
    int32_t start, rows, length, first;   // first row of q; rows (new tokens * group); tokens in the cache; position of the first new token
};

__device__ __forceinline__ Work work_of(const AttendArgs& a, uint32_t id)
{
    Work w;
    const uint32_t by_tile = divide(id, a.by_tiles), by_part = divide(by_tile, a.by_parts);
    w.tile = static_cast<int32_t>(id - by_tile * a.tiles);
    w.part = static_cast<int32_t>(by_tile - by_part * a.parts);
    w.sequence = static_cast<int32_t>(divide(by_part, a.by_heads));
    w.head = static_cast<int32_t>(by_part - w.sequence * a.kv_heads);
    const int32_t start = a.query_start[w.sequence], end = a.query_start[w.sequence + 1];
    w.start = min(max(start, 0), a.tokens);
    const int32_t count = min(max(end, w.start), a.tokens) - w.start;
    w.rows = count * a.group;
    w.length = static_cast<int32_t>(min(static_cast<int64_t>(max(a.lengths[w.sequence], 0)), static_cast<int64_t>(a.table_width) << a.page_shift));
    w.first = w.length - count;
    return w;
}

// Row of the parts' outputs of a new token's head.
__device__ __forceinline__ int64_t part_row_of(const AttendArgs& a, const Work& w, int32_t token, int32_t head)
{
    return (static_cast<int64_t>(w.part) * a.tokens + w.start + token) * a.q_heads + head;
}

// Keys that the rows [row, row + count) of a sequence see, cut to a part: [begin, end), begin a multiple of `block`.
struct Span {
    int32_t begin, end;
    int32_t low, high;   // positions of the first and the last row
    int32_t from;        // first key that any row sees

    // Whether some row does not see some of the keys [base, base + block).
    __device__ __forceinline__ bool edge(int32_t base, int32_t block, int32_t window) const
    {
        return base + block - 1 > low || base + block > end || (window > 0 && base <= high - window);
    }
};

__device__ __forceinline__ Span span_of(const AttendArgs& a, const Work& w, int32_t row, int32_t count, int32_t block)
{
    Span s;
    s.low = w.first + static_cast<int32_t>(divide(row, a.by_group));
    s.high = w.first + static_cast<int32_t>(divide(min(row + count, w.rows) - 1, a.by_group));
    s.from = a.window > 0 ? max(s.low - a.window + 1, 0) : 0;
    const int32_t to = s.high + 1;
    // 64 bits: parts beyond a short sequence's end
    const int64_t begin = s.from / block * block + static_cast<int64_t>(w.part) * a.per_part;
    s.begin = static_cast<int32_t>(min(begin, static_cast<int64_t>(max(to, 0))));
    s.end = w.part == static_cast<int32_t>(a.parts) - 1 ? to : static_cast<int32_t>(min(begin + a.per_part, static_cast<int64_t>(to)));
    return s;
}

// The page of a key as the table has it: what waits for the load is row_of.
__device__ __forceinline__ int32_t page_of(const AttendArgs& a, const int32_t* table, int32_t key) { return table[min(key >> a.page_shift, a.table_width - 1)]; }

// The same for a key that is the whole wavefront's, by a scalar load: it neither waits for the vector loads in flight nor they for it.
__device__ __forceinline__ int32_t shared_page_of(const AttendArgs& a, const int32_t* table, int32_t key)
{
    typedef const int32_t __attribute__((address_space(4))) * constant;
    return reinterpret_cast<constant>(reinterpret_cast<uintptr_t>(table))[__builtin_amdgcn_readfirstlane(min(key >> a.page_shift, a.table_width - 1))];
}

// Row of the pages where the 16 keys from `key` on lie; key is a multiple of 16, and so is a page.
__device__ __forceinline__ int64_t row_of(const AttendArgs& a, int32_t head, int32_t page, int32_t key)
{
    const uint32_t inside = min(static_cast<uint32_t>(max(page, 0)), static_cast<uint32_t>(a.pages - 1));
    return ((static_cast<int64_t>(inside) * a.kv_heads + head) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
}

__device__ __forceinline__ void load_eight(const void* p, int dtype, int64_t at, float (&f)[8])
{
    if (dtype == ACTQ_F32) {
        Eight<float> e;
        e.load(static_cast<const float*>(p) + at);
        e.widen(f);
    } else if (dtype == ACTQ_F16) {
        Eight<_Float16> e;
        e.load(static_cast<const _Float16*>(p) + at);
        e.widen(f);
    } else {
        Eight<__bf16> e;
        e.load(static_cast<const __bf16*>(p) + at);
        e.widen(f);
    }
}

template <int N>
__device__ __forceinline__ void store_some(void* p, int dtype, int64_t at, const float (&f)[N])
{
    static_assert(N % 4 == 0, "whole vectors");
    const auto put = [&](auto type) {
        typedef decltype(type) T;
        typedef T vector __attribute__((ext_vector_type(4)));
        typedef vector unaligned __attribute__((aligned(sizeof(T))));
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            vector v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = static_cast<T>(f[i + j]);
            *reinterpret_cast<unaligned*>(static_cast<T*>(p) + at + i) = v;
        }
    };
    if (dtype == ACTQ_F32) put(float{});
    else if (dtype == ACTQ_F16) put(_Float16{});
    else put(__bf16{});
}

// A number as it was rounded, which the operations on it see and not what it was computed from: a conversion of a product to binary16
// may become one instruction, which rounds once where a conversion of the rounded product rounds twice.
__device__ __forceinline__ float rounded(float v)
{
    asm("" : "+v"(v));
    return v;
}

// A number whose uses are computed where it is asked for: what is computed from a lane's number alone would otherwise be held in
// registers from the kernel's begin on, through the loop over the keys.
__device__ __forceinline__ int here(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

__device__ __forceinline__ int exponent(float v) { return static_cast<int>(bits_of(v) >> 23 & 255u) - 127; }

// The row of q that a lane has a share of: the exponent of its largest element, and whether one is no finite number.
struct RowScale {
    int exponent;
    bool bad;

    // With a cap, the cap in the row's unit has to stay a number.
    __device__ __forceinline__ RowScale(uint32_t largest, bool capped)
        : exponent(min(max(static_cast<int>(largest >> 23) - 127, capped ? -64 : -100), 126)), bad(largest >= 0x7f800000u) {}

    // An element as it goes to the matrix instructions, zero in a row that is none.
    __device__ __forceinline__ float scaled(float v) const { return bad ? 0.0f : ldexpf(v, kRowBits - exponent); }
    __device__ __forceinline__ float unit() const { return ldexpf(1.0f, exponent); }
};

__device__ __forceinline__ bool finite(float v) { return exponent(v) != 128; }

__device__ __forceinline__ bool is(float v, float constant) { return bits_of(v) == __builtin_bit_cast(uint32_t, constant); }

__device__ __forceinline__ float wave_max(float v)
{
    return over_lanes<64>(v, [](float a, float b) { return fmaxf(a, b); });
}

// tanh(x): for 16-bit outputs to 2^-21 of itself, from one exponential, whose cancellation below 1/2 a Pade approximant takes over (of order 5 over 4, off
// by 2^-33); both end in the same reciprocal, and no constant has to be held in a register.  For binary32 the function's own.
template <bool FINE>
__device__ __forceinline__ float tanh_of(float x)
{
    if (FINE) return tanhf(x);
    const float e = __builtin_amdgcn_exp2f(x * (2.0f * kLog2e)), u = x * x;
    const bool small = u < 0.25f;
    const float r = __builtin_amdgcn_rcpf(small ? fmaf(fmaf(15.0f, u, 420.0f), u, 945.0f) : e + 1.0f);
    return small ? x * fmaf(u + 105.0f, u, 945.0f) * r : fmaf(-2.0f, r, 1.0f);
}

// cap tanh(x / cap) of a score in units of a power of two, whose inverse is a matter of its exponent.
template <bool FINE>
__device__ __forceinline__ float capped(float x, float unit, float cap)
{
    return cap * __builtin_bit_cast(float, 0x7f000000u - __builtin_bit_cast(uint32_t, unit)) * tanh_of<FINE>(x * unit);
}

// f16 pair under zeros: byte B of `low` and of `high`.
template <int B>
__device__ __forceinline__ uint32_t byte_pair(uint32_t low, uint32_t high)
{
    return __builtin_amdgcn_perm(high, low, B | 0x0c00 | (4 + B) << 16 | 0x0c000000);
}

// Eight codes as subnormal binary16 numbers: two words of bytes, or one of nibbles, as pairs of nibble and nibble four further up
// (0 4 1 5 2 6 3 7).  Odd nibbles stay where they are, sixteen times as large; q has a sixteenth in their places.
__device__ __forceinline__ int code_order(int bits, int j) { return bits == 8 ? j : (j >> 1) + 4 * (j & 1); }
__device__ __forceinline__ int code_bits(int bits, int j) { return bits == 8 ? 0 : (j & 2) * 2; }   // to the left of where they belong

// CENTERED: (code - c) * 2^-9 instead, for binary32: scores are then sums of smaller terms, whose rounding is a third.
template <int BITS, bool CENTERED>
__device__ __forceinline__ f16x8 key_codes_of(const uint32_t* w)
{
    u32x4 r;
    if (BITS == 8) {
        r[0] = __builtin_amdgcn_perm(0, w[0], 0x0c010c00);
        r[1] = __builtin_amdgcn_perm(0, w[0], 0x0c030c02);
        r[2] = __builtin_amdgcn_perm(0, w[1], 0x0c010c00);
        r[3] = __builtin_amdgcn_perm(0, w[1], 0x0c030c02);
    } else {
        const uint32_t up = w[0] >> 8;
        r[0] = w[0] & 0x000f000fu;
        r[1] = w[0] & 0x00f000f0u;
        r[2] = up & 0x000f000fu;
        r[3] = up & 0x00f000f0u;
    }
    if (CENTERED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const _Float16 unit = BITS == 4 && i % 2 ? 2048.0f : 32768.0f, center = BITS == 8 ? -0.25f : -0.015625f;
            r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, uint32_t(r[i])), f16x2{unit, unit}, f16x2{center, center}));
        }
    }
    return __builtin_bit_cast(f16x8, r);
}

// Code pair of element I (of the words of two keys) as it lies: code * 2^-24, of odd nibbles code * 2^-20.
template <int BITS, int I>
__device__ __forceinline__ uint32_t raw_pair(const uint32_t* low, const uint32_t* high)
{
    if (BITS == 8) return byte_pair<I % 4>(low[I / 4], high[I / 4]);
    return byte_pair<I / 2 % 4>(low[I / 8], high[I / 8]) & (I % 2 ? 0x00f000f0u : 0x000f000fu);
}

// The same centred and scaled, (code - c) * 2^-9: exact in binary16.
template <int BITS, int I>
__device__ __forceinline__ f16x2 value_pair(const uint32_t* low, const uint32_t* high)
{
    const _Float16 unit = BITS == 4 && I % 2 ? 2048.0f : 32768.0f, center = BITS == 8 ? -0.25f : -0.015625f;
    return __builtin_elementwise_fma(__builtin_bit_cast(f16x2, raw_pair<BITS, I>(low, high)), f16x2{unit, unit}, f16x2{center, center});
}

// f(integral_constant 0), .., f(N - 1): a loop whose counter is a constant.
template <int N, typename F, int I = 0>
__device__ __forceinline__ void each(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, F, I + 1>(f);
    }
}

__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// A group's constants, lane by lane: scores are key * (q . codes) + key_zero * sum(q), in the row's unit; step and middle of the values.
struct Constants {
    float key, key_zero, step, middle;
};

// Constants of a key that some row sees, or (value header zero) of one that none does.  Where a value is no number, step is zero and
// middle is none: nothing times an infinity is no number either, so rows that see the key are made none on their own.
template <bool CENTERED>
__device__ __forceinline__ f32x4 constants_of(f32x2 key_header, f32x2 value_header, const AttendArgs& a, int key_bits, int value_bits)
{
    const float middle = fmaf(value_bits == 8 ? 128.0f : 8.0f, value_header[1], value_header[0]);
    const float zero = CENTERED ? fmaf(key_bits == 8 ? 128.0f : 8.0f, key_header[1], key_header[0]) : key_header[0];
    return f32x4{key_header[1] * a.factor * (CENTERED ? 1.0f / (1 << (kRowBits - kUnitBits)) : 1 << (24 - kRowBits)), zero * a.factor,
                 finite(middle) ? value_header[1] : 0.0f, middle};
}

// log2 of a key's step, or of a 128th of its middle, from above.
__device__ __forceinline__ float reach_of(const AttendArgs& a, float step, float middle)
{
    return fmaxf(static_cast<float>(exponent(fmaxf(fabsf(step), fabsf(middle) * 0.0078125f)) + 1), a.least);
}

// v * 2^x, where 2^x alone may be too small a number: the sums of two parts whose steps are 2^200 apart lie so far apart themselves.
struct Shrink {
    float half;
    __device__ __forceinline__ explicit Shrink(float x) : half(__builtin_amdgcn_exp2f(0.5f * x)) {}
    __device__ __forceinline__ float operator()(float v) const { return v * half * half; }
};

// ----------------------------------------------------------------------------- few rows

// Sixteen rows, whose keys four wavefronts share out in turn, blocks of 16 * TILES keys each.  Codes go from memory to the matrix
// instructions without the LDS: of a 16-key tile a lane loads its own pieces of one key, and for the values its own columns of eight
// keys, which it transposes itself as it widens them.  The next block's codes are loaded while one is computed.
constexpr int kFewWaves = 4;   // [8, which need no join up to 1024 keys: one token over 1021 11.0 -> 12.4 us]

// SPLIT: binary16 numbers for one of q, 1 for 16-bit types, 2 for binary32.
template <int DIM, int SPLIT, int KEY_BITS, int VALUE_BITS>
struct Few {
    static constexpr int kTiles = DIM == 256 ? 2 : 4, kBlock = 16 * kTiles;
    static constexpr int kSteps = DIM / 32;                              // of the first product
    static constexpr int kKeyBytes = DIM * KEY_BITS / 8;
    static constexpr int kPiece = kKeyBytes < 64 ? kKeyBytes / 4 : 16;   // bytes that a lane loads at once
    static constexpr int kPieces = kKeyBytes / 4 / kPiece;
    static constexpr int kPieceSteps = kPiece * 8 / KEY_BITS / 8;        // steps of the first product in a piece
    static constexpr int kColumns = DIM / 16;                            // of the values, per lane
    static constexpr int kValueBytes = kColumns * VALUE_BITS / 8;        // 2 to 16
    static constexpr int kValueWords = (kValueBytes + 3) / 4;

    struct Block {
        uint32_t key[kTiles][kPieces][kPiece / 4];
        uint32_t value[kTiles][4][kValueWords];   // [tile][key][word]
        f32x2 key_header, value_header;           // of the lane's own key
    };
};

template <int BYTES>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w)
{
    if constexpr (BYTES == 16) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else if constexpr (BYTES == 8) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p);
        w[0] = v[0];
        w[1] = v[1];
    } else if constexpr (BYTES == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
}

// WEIGHTS: binary16 numbers for a weight (by_numbers).
template <int DIM, int SPLIT, int WEIGHTS, int KEY_BITS, int VALUE_BITS>
__global__ __launch_bounds__(kFewWaves * 64, 2) void attend_few_kernel(AttendArgs a)
{
    typedef Few<DIM, SPLIT, KEY_BITS, VALUE_BITS> K;
    __shared__ float joined_out[kFewWaves / 2][K::kColumns][4][64];
    __shared__ float joined_max[kFewWaves][16], joined_sum[kFewWaves][16];
    const Work w = work_of(a, blockIdx.x);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int n = lane % 16, g = lane / 16;
    const int32_t* const table = a.table + static_cast<int64_t>(w.sequence) * a.table_width;
    for (int32_t tile = w.tile; 16 * static_cast<int64_t>(tile) < w.rows; tile += a.tiles) {
        const int32_t row = 16 * tile + n;
        const bool there = row < w.rows;
        const int32_t token = static_cast<int32_t>(divide(there ? row : w.rows - 1, a.by_group));
        const int32_t head = w.head * a.group + (there ? row : w.rows - 1) - token * a.group;
        const int32_t position = w.first + token;
        const Span span = span_of(a, w, 16 * tile, 16, K::kBlock);
        if (a.partial && span.begin >= span.end) {   // a part beyond a short sequence's end
            if (threadIdx.x < 16 && there) a.partial_sums[part_row_of(a, w, token, head)] = f32x2{kNothing, 0.0f};
            continue;
        }

        // pages of a block, whose look-up is not waited for; then its codes: rows of the pages are the wavefront's, places in them the lane's
        int32_t pages[K::kTiles];
        const auto find = [&](int32_t base) {
#pragma unroll
            for (int t = 0; t < K::kTiles; ++t) pages[t] = shared_page_of(a, table, base + 16 * t);
        };
        const uint32_t key_place = n * K::kKeyBytes + g * K::kPiece, value_place = 4 * g * (DIM / 8 * VALUE_BITS) + n * K::kValueBytes;
        const auto load = [&](typename K::Block& b, int32_t base) {
            int64_t rows[K::kTiles];
#pragma unroll
            for (int t = 0; t < K::kTiles; ++t) rows[t] = row_of(a, w.head, pages[t], base + 16 * t);
            // the lane's own key: number n % 4 of group g's four of tile n / 4
            int64_t own = rows[0];
#pragma unroll
            for (int t = 1; t < K::kTiles; ++t) own = n / 4 % K::kTiles == t ? rows[t] : own;
            own += 4 * g + n % 4;
            b.key_header = *reinterpret_cast<const f32x2*>(a.key_header + 2 * own);
            b.value_header = *reinterpret_cast<const f32x2*>(a.value_header + 2 * own);
#pragma unroll
            for (int t = 0; t < K::kTiles; ++t) {
                const uint8_t* const p = a.key_codes + rows[t] * K::kKeyBytes;
#pragma unroll
                for (int i = 0; i < K::kPieces; ++i) load_words<K::kPiece>(p + key_place + 4 * i * K::kPiece, b.key[t][i]);
            }
#pragma unroll
            for (int t = 0; t < K::kTiles; ++t) {
                const uint8_t* const p = a.value_codes + rows[t] * (DIM / 8 * VALUE_BITS);
#pragma unroll
                for (int k = 0; k < 4; ++k) load_words<K::kValueBytes>(p + value_place + k * (DIM / 8 * VALUE_BITS), b.value[t][k]);
            }
        };

        // the first block is on its way before q is asked for: a workgroup's begin is a chain of trips to memory
        int32_t base = span.begin + wave * K::kBlock;
        constexpr int32_t kStride = kFewWaves * K::kBlock;
        typename K::Block now;
        if (base < span.end) {
            find(base);
            load(now, base);
            find(min(base + kStride, span.end - 1));
        }

        // q, a lane's 8 elements of its row for every step
        f16x8 q[SPLIT][K::kSteps];
        float q_sum = 0.0f, unit, sum;
        {
            const int64_t at = (static_cast<int64_t>(w.start) + token) * a.q.token + head * a.q.head;
            float f[K::kSteps][8];
            uint32_t largest = 0;
#pragma unroll
            for (int s = 0; s < K::kSteps; ++s) {
                const int piece = s / K::kPieceSteps, in_piece = s % K::kPieceSteps;
                load_eight(a.q.p, a.dtype, at + (4 * piece + g) * (8 * K::kPieceSteps) + 8 * in_piece, f[s]);
#pragma unroll
                for (int j = 0; j < 8; ++j) largest = max(largest, magnitude(f[s][j]));
            }
            largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 16)));
            largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 32)));
            const RowScale row_scale(largest, a.cap > 0.0f);
#pragma unroll
            for (int s = 0; s < K::kSteps; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float whole = row_scale.scaled(f[s][code_order(KEY_BITS, j)]);
                    q_sum += whole;
                    const float v = ldexpf(whole, SPLIT == 2 ? 0 : -code_bits(KEY_BITS, j));
                    q[0][s][j] = static_cast<_Float16>(v);
                    if (SPLIT == 2) q[SPLIT - 1][s][j] = static_cast<_Float16>(v - static_cast<float>(q[0][s][j]));
                }
            q_sum += __shfl_xor(q_sum, 16);
            q_sum += __shfl_xor(q_sum, 32);
            q_sum *= 1.0f / (1 << kRowBits);
            unit = row_scale.unit();
            sum = nan_where(row_scale.bad && position >= 0);   // a row that sees something and is not finite
        }

        float m = kNothing, middle = 0.0f;
        float ceiling = a.least;   // the largest reach of the wavefront's keys so far
        f32x4 acc[K::kColumns];
#pragma unroll
        for (int i = 0; i < K::kColumns; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // Codes are multiplied as they lie and centred at the end, by the sum of the very weights that they were multiplied with: one product
        // more for one instruction less per pair of codes.  The sums are larger than centred ones, by 2.5 where a group is normal, and so is
        // their rounding: far below that of a 16-bit result, but not for binary32, whose codes are centred at once.
        f32x4 weights = {0.0f, 0.0f, 0.0f, 0.0f};
        const _Float16 one = 1.0f;
        const f16x8 ones = {one, one, one, one, one, one, one, one};

        const auto use = [&](const typename K::Block& b, int32_t base) {
            const int32_t own = base + 16 * (n / 4 % K::kTiles) + 4 * g + n % 4;
            const bool seen = own >= span.from && own < span.end;   // by any row
            const f32x2 value_header = {seen ? b.value_header[0] : 0.0f, seen ? b.value_header[1] : 0.0f};
            const f32x4 four = constants_of<SPLIT == 2>(b.key_header, value_header, a, KEY_BITS, VALUE_BITS);
            Constants c = {four[0], four[1], four[2], four[3]};
            const bool bad = !finite(c.middle);
            const float reach = reach_of(a, c.step, bad ? 0.0f : c.middle);
            if (__any(reach > ceiling)) ceiling = wave_max(reach);
            settled(c.key_zero);
            f32x4 x[K::kTiles];
#pragma unroll
            for (int t = 0; t < K::kTiles; ++t) {
                x[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < K::kSteps; ++s) {
                    const f16x8 codes = key_codes_of<KEY_BITS, SPLIT == 2>(&b.key[t][s / K::kPieceSteps][s % K::kPieceSteps * (KEY_BITS / 4)]);
#pragma unroll
                    for (int h = 0; h < SPLIT; ++h) x[t] = multiply(codes, q[h][s], x[t]);
                }
            }
            float top = kNothing;
            each<K::kTiles>([&](auto t) {
                each<4>([&](auto e) {
                    constexpr int i = e, kAt = kDppBroadcast + 4 * t + i;
                    x[t][i] = add_broadcast<4 * t + i>(dpp<kAt>(c.key) * x[t][i], c.key_zero, q_sum, q_sum);
                });
            });
            if (a.cap > 0.0f) {
#pragma unroll
                for (int t = 0; t < K::kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][i] = capped<SPLIT == 2>(x[t][i], unit, a.cap);
            }
            // f(tile, i, whether the row sees key i of it): key = base + 4 g + a constant, between the window's begin and the last one in sight
            const auto each_key = [&](auto f) {
                const int32_t last = min(position, span.end - 1) - base - 4 * g, before = a.window > 0 ? position - a.window - base - 4 * g : -1;
                each<K::kTiles>([&](auto t) { each<4>([&](auto e) { f(t, e, 16 * t + e <= last && 16 * t + e > before); }); });
            };
            if (span.edge(base, K::kBlock, a.window)) {
                each_key([&](auto t, auto e, bool sees) {
                    constexpr int i = e;
                    x[t][i] = sees ? x[t][i] : -INFINITY;
                });
            }
#pragma unroll
            for (int t = 0; t < K::kTiles; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, x[t][i]);
            top *= unit;
            if (__any(top + ceiling > m + kMostWeight)) {
                float peak = kNothing;
                each<K::kTiles>([&](auto t) {
                    each<4>([&](auto e) {
                        constexpr int i = e;
                        peak = fmaxf(peak, fmaf(x[t][i], unit, dpp<kDppBroadcast + 4 * t + i>(reach)));
                    });
                });
                peak = fmaxf(peak, __shfl_xor(peak, 16));
                peak = fmaxf(peak, __shfl_xor(peak, 32));
                const float now = peak > m + kMostWeight ? peak - kNewWeight : m;   // a row's doing alone
                const Shrink less(m - now);
                m = now;
                sum = less(sum);
                middle = less(middle);
#pragma unroll
                for (int i = 0; i < K::kColumns; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][r] = less(acc[i][r]);
                weights[0] = less(weights[0]);
            }
            if (__any(bad)) {
                each_key([&](auto t, auto e, bool sees) {
                    const float none = dpp<kDppBroadcast + 4 * t + e>(nan_where(bad));
                    sum += sees ? none : 0.0f;
                });
                c.middle = bad ? 0.0f : c.middle;
            }
            settled(c.middle);
            f16x8 p[WEIGHTS][K::kTiles / 2];
            float block_sum = 0.0f, block_middle = 0.0f;   // of the block first: one sum over thousands of keys would gather their roundings
            each<K::kTiles>([&](auto t) {
                each<4>([&](auto e) {
                    constexpr int i = e, kAt = kDppBroadcast + 4 * t + i;
                    const float v = __builtin_amdgcn_exp2f(fmaf(x[t][i], unit, -m));
                    block_sum += v;
                    const float weight = WEIGHTS == 2 ? rounded(dpp<kAt>(c.step) * v) : dpp<kAt>(c.step) * v;   // the same one for both of its numbers
                    block_middle = add_broadcast<4 * t + i>(block_middle, c.middle, v, weight);
                    const _Float16 high = static_cast<_Float16>(weight);
                    p[0][t / 2][4 * (t % 2) + i] = high;
                    if (WEIGHTS == 2) p[WEIGHTS - 1][t / 2][4 * (t % 2) + i] = static_cast<_Float16>(weight - static_cast<float>(high));
                });
            });
            sum += block_sum;
            middle += block_middle;
            if (SPLIT == 1) {
#pragma unroll
                for (int s = 0; s < K::kTiles / 2; ++s)
#pragma unroll
                    for (int h = 0; h < WEIGHTS; ++h) weights = multiply(ones, p[h][s], weights);
            }
#pragma unroll
            for (int s = 0; s < K::kTiles / 2; ++s)
                each<K::kColumns>([&](auto i) {
                    f16x8 values;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t (&key)[4][K::kValueWords] = b.value[2 * s + k / 2];
                        const uint32_t *const low = key[2 * (k % 2)], *const high = key[2 * (k % 2) + 1];
                        const f16x2 pair = SPLIT == 2 ? value_pair<VALUE_BITS, i>(low, high) : __builtin_bit_cast(f16x2, raw_pair<VALUE_BITS, i>(low, high));
                        values[2 * k] = pair[0];
                        values[2 * k + 1] = pair[1];
                    }
#pragma unroll
                    for (int h = 0; h < WEIGHTS; ++h) acc[i] = multiply(values, p[h][s], acc[i]);
                });
        };

        if (base < span.end) {
            typename K::Block next;
            while (true) {
                const int32_t after = base + kStride;
                if (after < span.end) {
                    load(next, after);
                    find(min(after + kStride, span.end - 1));
                }
                use(now, base);
                if (after >= span.end) break;
                now = next;
                base = after;
            }
        }

        // the wavefronts' shares: a row's maximum and sum first, then the outputs in two steps through the LDS
        const int place = here(lane);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        middle += __shfl_xor(middle, 16);
        middle += __shfl_xor(middle, 32);
        if (g == 0) {
            joined_max[wave][n] = m;
            joined_sum[wave][n] = sum;
        }
        __syncthreads();
        float top = joined_max[0][n];
#pragma unroll
        for (int k = 1; k < kFewWaves; ++k) top = fmaxf(top, joined_max[k][n]);
        float total = 0.0f;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) total += Shrink(joined_max[k][n] - top)(joined_sum[k][n]);
        const Shrink share(m - top);
#pragma unroll
        for (int i = 0; i < K::kColumns; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int unit = SPLIT == 2 ? kUnitBits : VALUE_BITS == 4 && i % 2 ? 20 : 24;
                const float centered = SPLIT == 2 ? acc[i][r] : fmaf(weights[0], (VALUE_BITS == 8 ? -128.0f : -8.0f) / (1 << unit), acc[i][r]);
                acc[i][r] = share(fmaf(centered, static_cast<float>(1 << unit), middle));
            }
#pragma unroll
        for (int step = kFewWaves / 2; step >= 1; step /= 2) {
            if (wave >= step && wave < 2 * step) {
#pragma unroll
                for (int i = 0; i < K::kColumns; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) joined_out[wave - step][i][r][place] = acc[i][r];
            }
            __syncthreads();
            if (wave < step) {
#pragma unroll
                for (int i = 0; i < K::kColumns; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][r] += joined_out[wave][i][r][place];
            }
            __syncthreads();   // read before the next step writes there
        }
        if (wave == 0 && there) {
            const float scale = is(total, 0.0f) ? 0.0f : 1.0f / total;   // nothing in sight: zeros
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float f[K::kColumns];
#pragma unroll
                for (int i = 0; i < K::kColumns; ++i) f[i] = acc[i][r] * scale;
                const int at = K::kColumns * (4 * (place / 16) + r);
                if (a.partial) store_some(a.partial, ACTQ_F32, part_row_of(a, w, token, head) * DIM + at, f);
                else store_some(a.out.p, a.dtype, (static_cast<int64_t>(w.start) + token) * a.out.token + head * a.out.head + at, f);
            }
            if (a.partial && g == 0) a.partial_sums[part_row_of(a, w, token, head)] = f32x2{top, total};
        }
    }
}

// ----------------------------------------------------------------------------- many rows

// 32 rows per wavefront, WAVES of them over the same keys.  Tiles of keys are widened once per workgroup into the LDS (keys as
// they lie, values transposed), twice buffered: while one is computed the next one's codes are on their way to registers.  Half of the wavefronts
// widen keys and half values; the last one prepares the groups' constants.
//
// The 32 x 32 product gives a lane the scores of its row (lane % 32) for the keys 8 (i / 4) + 4 (lane / 32) + i % 4, i = 0..15; two
// steps of the second product take eight of them each, and the transposed values hold a step's sixteen keys in that order.
// Rows of the LDS are 16-byte chunks; a chunk's place is its number XOR some bits of the row, so that neither the rows that eight lanes read
// together nor those that they write share a bank.  Of sixteen neighbouring codes of a key the first eight go to the row's first half.
template <int DIM, int SPLIT, int WAVES>
struct Many {
    static constexpr int kThreads = 64 * WAVES, kOwnRows = 32, kRows = kOwnRows * WAVES;
    static constexpr int kTile = 8192 / DIM;           // keys of a tile
    static constexpr int kParts = kTile / 32;          // of 32 keys
    static constexpr int kSteps = DIM / 16;            // of the first product
    static constexpr int kBlocks = DIM / 32;           // of the outputs
    static constexpr int kHalf = kThreads / 2;         // threads that widen keys, and values
    static constexpr int kKeyUnits = 512 / kHalf;      // a unit: 16 codes of a key
    static constexpr int kValueUnits = 256 / kHalf;    // a unit: 8 columns of 4 keys
    static constexpr int kOwn = kTile > 64 ? 2 : 1;    // groups of a lane whose constants it prepares
    static constexpr int kChunks = kTile / 8;          // of a row of values

    __device__ static __forceinline__ int key_place(int key, int chunk) { return key * (DIM * 2) + ((chunk ^ (key & 7)) << 4); }
    __device__ static __forceinline__ int value_place(int column, int chunk)
    {
        const int x = kChunks >= 8 ? (column ^ (column >> 3 & 3)) & 7 : (column >> 1 ^ column >> 3) & 3;
        return column * (kTile * 2) + ((chunk ^ x) << 4);
    }
};

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DIM, int SPLIT, int WEIGHTS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 ? 2 : 1) void attend_many_kernel(AttendArgs a)
{
    typedef Many<DIM, SPLIT, WAVES> K;
    __shared__ __attribute__((aligned(16))) uint8_t keys[2][16384];
    __shared__ __attribute__((aligned(16))) uint8_t values[2][16384];
    __shared__ f32x4 constants[2][K::kTile];   // as in Constants
    __shared__ float ceilings[2];   // the largest reach of the tile's keys

    const Work w = work_of(a, blockIdx.x);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int n = lane % 32, h = lane / 32;
    const int32_t* const table = a.table + static_cast<int64_t>(w.sequence) * a.table_width;
    const bool of_values = wave < WAVES / 2, of_constants = wave == WAVES - 1;
    const int unit = threadIdx.x % K::kHalf;
    constexpr std::integral_constant<int, 8> eight;
    constexpr std::integral_constant<int, 4> four;
    // two wavefronts share a SIMD: one goes ahead, so that one's products meet the other's softmax
    if (WAVES == 8 && wave >= WAVES / 2) __builtin_amdgcn_s_setprio(1);

    // the thread's units: keys 16 codes (chunk, key), values 8 columns of 4 keys
    const auto key_of = [&](int u) { return (unit + u * K::kHalf) / (DIM / 16); };
    const auto chunk_of = [&](int u) { return (unit + u * K::kHalf) % (DIM / 16); };
    // a unit's bits, low ones first, so that sixteen lanes write all banks: half of a chunk, two bits of the columns, the upper bit of the step ..
    const auto bit = [&](int u, int i) { return (unit + u * K::kHalf) >> i & 1; };
    const auto half_of = [&](int u) { return bit(u, 0); };   // the four keys are quad 2 half + odd of a step's
    const auto odd_of = [&](int u) { return bit(u, DIM == 256 ? 3 : 5); };
    const auto columns_of = [&](int u) {
        return bit(u, 1) + 2 * bit(u, 2) + 4 * bit(u, 4) + (DIM == 64 ? 0 : DIM == 128 ? 8 * bit(u, 7) : 8 * bit(u, 6) + 16 * bit(u, 7));
    };
    const auto step_of = [&](int u) { return DIM == 256 ? bit(u, 5) : bit(u, 6) + 2 * bit(u, 3) + (DIM == 64 ? 4 * bit(u, 7) : 0); };
    // where the lane reads: of the first step, the others' chunks by XOR, blocks of 32 columns by their distance
    const int key_at = K::key_place(n, h), value_at = K::value_place(n, h);

    for (int32_t tile = static_cast<int32_t>(a.tiles) - 1 - w.tile; K::kRows * static_cast<int64_t>(tile) < w.rows; tile += a.tiles) {
        const int32_t first_row = K::kRows * tile + K::kOwnRows * wave;
        const bool any = first_row < w.rows;
        const Span span = span_of(a, w, K::kRows * tile, K::kRows, K::kTile);
        if (a.partial && span.begin >= span.end) {   // a part beyond a short sequence's end
            for (int r = threadIdx.x; r < K::kRows && K::kRows * tile + r < w.rows; r += K::kThreads) {
                const int32_t token = static_cast<int32_t>(divide(K::kRows * tile + r, a.by_group));
                a.partial_sums[part_row_of(a, w, token, w.head * a.group + K::kRows * tile + r - token * a.group)] = f32x2{kNothing, 0.0f};
            }
            continue;
        }
        Span mine = span;   // of the wavefront's rows
        if (any) {
            mine.low = w.first + static_cast<int32_t>(divide(first_row, a.by_group));
            mine.high = w.first + static_cast<int32_t>(divide(min(first_row + K::kOwnRows, w.rows) - 1, a.by_group));
            mine.from = a.window > 0 ? max(mine.low - a.window + 1, 0) : 0;
        }
        // the lane's row; beyond the last one the last one again
        const auto token_of_row = [&] { return static_cast<int32_t>(divide(min(first_row + n, w.rows - 1), a.by_group)); };
        const auto head_of_row = [&] { return w.head * a.group + min(first_row + n, w.rows - 1) - token_of_row() * a.group; };

        int32_t pages[K::kKeyUnits], own_pages[K::kOwn];
        uint32_t codes[8 * K::kValueUnits];
        f32x2 key_header[K::kOwn], value_header[K::kOwn];

        // pages of a tile, then its codes, then the LDS
        const auto find = [&](int32_t base) {
            if (of_values) {
#pragma unroll
                for (int u = 0; u < K::kValueUnits; ++u) pages[u] = page_of(a, table, base + 16 * step_of(u));
            } else {
#pragma unroll
                for (int u = 0; u < K::kKeyUnits; ++u) pages[u] = page_of(a, table, base + key_of(u));
            }
            if (of_constants) {
#pragma unroll
                for (int o = 0; o < K::kOwn; ++o) own_pages[o] = page_of(a, table, base + (lane + 64 * o) % K::kTile);
            }
        };
        const auto load = [&](int32_t base) {
            const auto load_values = [&](auto bits) {
                constexpr int kBits = decltype(bits)::value, kBytes = DIM / 8 * kBits;
#pragma unroll
                for (int u = 0; u < K::kValueUnits; ++u) {
                    const uint8_t* const p = a.value_codes + (row_of(a, w.head, pages[u], base + 16 * step_of(u)) + 8 * half_of(u) + 4 * odd_of(u)) * kBytes + columns_of(u) * kBits;
#pragma unroll
                    for (int k = 0; k < 4; ++k) load_words<kBits>(p + k * kBytes, codes + 8 * u + 2 * k);
                }
            };
            const auto load_keys = [&](auto bits) {
                constexpr int kBits = decltype(bits)::value, kBytes = DIM / 8 * kBits;
#pragma unroll
                for (int u = 0; u < K::kKeyUnits; ++u)
                    load_words<2 * kBits>(a.key_codes + row_of(a, w.head, pages[u], base + key_of(u)) * kBytes + chunk_of(u) * 2 * kBits, codes + 4 * u);
            };
            if (of_values) a.value_bits == 8 ? load_values(eight) : load_values(four);
            else a.key_bits == 8 ? load_keys(eight) : load_keys(four);
            if (of_constants) {
#pragma unroll
                for (int o = 0; o < K::kOwn; ++o) {
                    const int64_t own = row_of(a, w.head, own_pages[o], base + (lane + 64 * o) % K::kTile);
                    key_header[o] = *reinterpret_cast<const f32x2*>(a.key_header + 2 * own);
                    value_header[o] = *reinterpret_cast<const f32x2*>(a.value_header + 2 * own);
                }
            }
        };
        // the first tile is on its way before q is asked for: a workgroup's begin is a chain of trips to memory
        const int32_t last = span.end - 1;
        if (span.begin < span.end) {
            find(span.begin);
            load(span.begin);
            find(min(span.begin + K::kTile, last));
        }

        // q, a lane's 8 elements of its rows for every step
        f16x8 q[SPLIT][K::kSteps];
        float q_sum, unit, sum;
        {
            // element of q in slot 0 of a step: the order of the chunks in the LDS
            const auto at = [&](int s) {
                const int chunk = 2 * s + h;
                return (static_cast<int64_t>(w.start) + token_of_row()) * a.q.token + head_of_row() * a.q.head + (chunk < DIM / 16 ? 16 * chunk : 16 * chunk - DIM + 8);
            };
            uint32_t largest = 0;
#pragma unroll
            for (int s = 0; s < K::kSteps; ++s) {
                float f[8];
                load_eight(a.q.p, a.dtype, at(s), f);
#pragma unroll
                for (int j = 0; j < 8; ++j) largest = max(largest, magnitude(f[j]));
            }
            largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 32)));
            const RowScale row_scale(largest, a.cap > 0.0f);
            q_sum = 0.0f;
            // once more, from the cache: held until here they would be twice the registers of everything else
#pragma unroll
            for (int s = 0; s < K::kSteps; ++s) {
                float f[8];
                load_eight(a.q.p, a.dtype, at(s), f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = row_scale.scaled(f[j]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    q_sum += f[j];
                    const float v = ldexpf(a.key_bits == 8 ? f[j] : f[code_order(4, j)], a.key_bits == 8 || SPLIT == 2 ? 0 : -code_bits(4, j));
                    q[0][s][j] = static_cast<_Float16>(v);
                    if (SPLIT == 2) q[SPLIT - 1][s][j] = static_cast<_Float16>(v - static_cast<float>(q[0][s][j]));
                }
            }
            q_sum += __shfl_xor(q_sum, 32);
            q_sum *= 1.0f / (1 << kRowBits);
            unit = row_scale.unit();
            sum = nan_where(row_scale.bad && w.first + token_of_row() >= 0);   // a row that sees something and is not finite
        }

        float m = kNothing, middle = 0.0f;
        f32x16 acc[K::kBlocks];
#pragma unroll
        for (int b = 0; b < K::kBlocks; ++b) acc[b] = f32x16{};

        const auto store = [&](int32_t base, int to) {
            const auto store_values = [&](auto bits) {
                constexpr int kBits = decltype(bits)::value;
#pragma unroll
                for (int u = 0; u < K::kValueUnits; ++u) {
                    const int chunk = 2 * step_of(u) + odd_of(u), half = 8 * half_of(u);
                    const uint32_t* const c = codes + 8 * u;
                    each<8>([&](auto i) {
                        const u32x2 both = {__builtin_bit_cast(uint32_t, value_pair<kBits, i>(c, c + 2)), __builtin_bit_cast(uint32_t, value_pair<kBits, i>(c + 4, c + 6))};
                        *reinterpret_cast<u32x2*>(&values[to][K::value_place(8 * columns_of(u) + i, chunk) + half]) = both;
                    });
                }
            };
            const auto store_keys = [&](auto bits) {
                constexpr int kBits = decltype(bits)::value;
#pragma unroll
                for (int u = 0; u < K::kKeyUnits; ++u) {
                    *reinterpret_cast<f16x8*>(&keys[to][K::key_place(key_of(u), chunk_of(u))]) = key_codes_of<kBits, SPLIT == 2>(codes + 4 * u);
                    *reinterpret_cast<f16x8*>(&keys[to][K::key_place(key_of(u), chunk_of(u) + DIM / 16)]) = key_codes_of<kBits, SPLIT == 2>(codes + 4 * u + kBits / 4);
                }
            };
            if (of_values) a.value_bits == 8 ? store_values(eight) : store_values(four);
            else a.key_bits == 8 ? store_keys(eight) : store_keys(four);
            if (of_constants) {
                float top = a.least;
#pragma unroll
                for (int o = 0; o < K::kOwn; ++o) {
                    const int32_t own = base + (lane + 64 * o) % K::kTile;
                    const bool seen = own >= span.from && own < span.end;   // by any row
                    const f32x2 header = {seen ? value_header[o][0] : 0.0f, seen ? value_header[o][1] : 0.0f};
                    const f32x4 c = constants_of<SPLIT == 2>(key_header[o], header, a, a.key_bits, a.value_bits);
                    top = fmaxf(top, reach_of(a, c[2], finite(c[3]) ? c[3] : 0.0f));
                    if (lane + 64 * o < K::kTile) constants[to][lane + 64 * o] = c;
                }
                top = wave_max(top);
                if (lane == 0) ceilings[to] = top;
            }
        };

        // keys of part s of the tile in buffer `from`, all on their way before the first product: left to itself the compiler waits for each
        f16x8 c_keys[K::kSteps];
        const auto load_part = [&](int from, int s) {
#pragma unroll
            for (int k = 0; k < K::kSteps; ++k) c_keys[k] = *reinterpret_cast<const f16x8*>(&keys[from][0] + (key_at + s * (64 * DIM) ^ k << 5));
        };

        // Scores and sums of the keys [base, base + 32), that part; the next part's keys are loaded behind the products that need these.
        const auto use = [&](int32_t base, int from, int s, bool more) {
            const f32x4 v = constants[from][32 * s + 8 * (lane % 16 / 4) + 4 * h + lane % 4];
            const float ceiling = ceilings[from];
            __builtin_amdgcn_sched_barrier(0);
            f32x16 x = {};
#pragma unroll
            for (int k = 0; k < K::kSteps; ++k)
#pragma unroll
                for (int i = 0; i < SPLIT; ++i) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(c_keys[k], q[i][k], x, 0, 0, 0);
            f16x8 u[K::kBlocks][2];
#pragma unroll
            for (int b = 0; b < K::kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 2; ++k) u[b][k] = *reinterpret_cast<const f16x8*>(&values[from][0] + (value_at ^ (2 * s + k) << 5) + b * (64 * K::kTile));
            Constants c = {v[0], v[1], v[2], v[3]};
            settled(c.key_zero);
            each<16>([&](auto e) {
                constexpr int i = e, kAt = kDppBroadcast + i;
                x[i] = add_broadcast<i>(dpp<kAt>(c.key) * x[i], c.key_zero, q_sum, q_sum);
            });
            if (a.cap > 0.0f) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = capped<SPLIT == 2>(x[i], unit, a.cap);
            }
            // f(i, whether the row sees key i): key = base + 4 h + a constant, between the window's begin and the last one in sight
            const auto each_key = [&](auto f) {
                const int32_t position = w.first + token_of_row();
                const int32_t last = min(position, span.end - 1) - base - 4 * h, before = a.window > 0 ? position - a.window - base - 4 * h : -1;
                each<16>([&](auto e) {
                    constexpr int kKey = 8 * (e / 4) + e % 4;
                    f(e, kKey <= last && kKey > before);
                });
            };
            if (mine.edge(base, 32, a.window)) {
                each_key([&](auto e, bool sees) {
                    constexpr int i = e;
                    x[i] = sees ? x[i] : -INFINITY;
                });
            }
            float top = kNothing;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
            top *= unit;
            if (__any(top + ceiling > m + kMostWeight)) {
                const float reach = reach_of(a, c.step, finite(c.middle) ? c.middle : 0.0f);
                float peak = kNothing;
                each<16>([&](auto e) {
                    constexpr int i = e;
                    peak = fmaxf(peak, fmaf(x[i], unit, dpp<kDppBroadcast + i>(reach)));
                });
                peak = fmaxf(peak, __shfl_xor(peak, 32));
                const float now = peak > m + kMostWeight ? peak - kNewWeight : m;   // a row's doing alone
                const Shrink less(m - now);
                m = now;
                sum = less(sum);
                middle = less(middle);
#pragma unroll
                for (int b = 0; b < K::kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[b][i] = less(acc[b][i]);
            }
            const bool bad = !finite(c.middle);
            if (__any(bad)) {
                each_key([&](auto e, bool sees) {
                    const float none = dpp<kDppBroadcast + e>(nan_where(bad));
                    sum += sees ? none : 0.0f;
                });
                c.middle = bad ? 0.0f : c.middle;
            }
            settled(c.middle);
            if (more) load_part(from, s + 1);
            f16x8 p[WEIGHTS][2];
            float part_sum = 0.0f, part_middle = 0.0f;   // of the part first: one sum over thousands of keys would gather their roundings
            each<16>([&](auto e) {
                constexpr int i = e, kAt = kDppBroadcast + i;
                const float v = __builtin_amdgcn_exp2f(fmaf(x[i], unit, -m));
                part_sum += v;
                const float weight = WEIGHTS == 2 ? rounded(dpp<kAt>(c.step) * v) : dpp<kAt>(c.step) * v;   // the same one for both of its numbers
                part_middle = add_broadcast<i>(part_middle, c.middle, v, weight);
                const _Float16 high = static_cast<_Float16>(weight);
                p[0][i / 8][i % 8] = high;
                if (WEIGHTS == 2) p[WEIGHTS - 1][i / 8][i % 8] = static_cast<_Float16>(weight - static_cast<float>(high));
            });
            sum += part_sum;
            middle += part_middle;
#pragma unroll
            for (int b = 0; b < K::kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < WEIGHTS; ++i) acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(u[b][k], p[i][k], acc[b], 0, 0, 0);
        };

        if (span.begin < span.end) {
            store(span.begin, 0);
            if (span.begin + K::kTile < span.end) load(span.begin + K::kTile);
            find(min(span.begin + 2 * K::kTile, last));
            __syncthreads();
            int at = 0;
            for (int32_t base = span.begin; base < span.end; base += K::kTile, at ^= 1) {
                // the next tile from the registers to the LDS, the one after it on its way to them
                const auto stage = [&] {
                    if (base + K::kTile < span.end) store(base + K::kTile, at ^ 1);
                    if (base + 2 * K::kTile < span.end) {
                        load(base + 2 * K::kTile);
                        find(min(base + 3 * K::kTile, last));
                    }
                };
                if (of_values) stage();
                if (any && base <= mine.high && base + K::kTile > mine.from) {
                    // the parts that some row sees
                    const int s_begin = max(mine.from - base, 0) / 32, s_end = min((min(mine.high + 1, span.end) - base + 31) / 32, K::kParts);
                    if (s_begin < s_end) load_part(at, s_begin);
                    for (int s = s_begin; s < s_end; ++s) use(base + 32 * s, at, s, s + 1 < s_end);
                }
                if (!of_values) stage();   // behind the products where the others stage ahead of them
                __syncthreads();
            }
        }

        sum += __shfl_xor(sum, 32);
        middle += __shfl_xor(middle, 32);
        if (first_row + n < w.rows) {
            const float scale = is(sum, 0.0f) ? 0.0f : 1.0f / sum;   // nothing in sight: zeros
            const int32_t token = token_of_row(), head = head_of_row();
            const int64_t part_row = part_row_of(a, w, token, head);
#pragma unroll
            for (int b = 0; b < K::kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    float f[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = fmaf(acc[b][i + j], static_cast<float>(1 << kUnitBits), middle) * scale;
                    const int column = 32 * b + 2 * i + 4 * (here(lane) / 32);
                    if (a.partial) store_some(a.partial, ACTQ_F32, part_row * DIM + column, f);
                    else store_some(a.out.p, a.dtype, (static_cast<int64_t>(w.start) + token) * a.out.token + head * a.out.head + column, f);
                }
            if (a.partial && h == 0) a.partial_sums[part_row] = f32x2{m, sum};
        }
        __syncthreads();   // the next tile writes the LDS again
    }
}

// ----------------------------------------------------------------------------- joining parts

// A workgroup per row: the parts' outputs weighted by their sums at the largest maximum.  DIM / 4 threads take a part, four columns each, the others the
// next ones, with four parts' loads in flight; their sums meet in the LDS.  In a loop of one wavefront a part costs a trip to memory, 1.2 us.
constexpr int kJoinThreads = 256;
constexpr int kMostParts = 128;

// SHARED: all teams share a row; else each has its own, which is faster below kSharedParts parts (own -> shared, us of both kernels: one sequence, 32 rows of
// 128, 2 parts 11.0 -> 11.3, 4 parts 11.1 -> 11.5, 8 parts 11.8 -> 11.6, 15 parts 13.2 -> 12.1; four sequences 4 parts 11.8 -> 12.0, 8 parts 12.7 -> 12.3).
constexpr int kSharedParts = 8;

template <int DIM, bool SHARED>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendArgs a)
{
    constexpr int kColumns = DIM / 4, kTeams = kJoinThreads / kColumns, kAhead = 4, kStride = SHARED ? kTeams : 1;
    __shared__ float weights[SHARED ? 1 : kTeams][SHARED ? kMostParts : kSharedParts];
    __shared__ f32x4 sums[SHARED ? kTeams : 1][kColumns];
    __shared__ float tops[kJoinThreads / 64];
    const int64_t rows = static_cast<int64_t>(a.tokens) * a.q_heads;
    const int column = threadIdx.x % kColumns, team = threadIdx.x / kColumns, parts = static_cast<int>(a.parts);
    const int64_t row = SHARED ? static_cast<int64_t>(blockIdx.x) : static_cast<int64_t>(blockIdx.x) * kTeams + team;
    const bool there = row < rows;
    const int own = SHARED ? static_cast<int>(threadIdx.x) : column;   // the part whose weight the thread works out
    const f32x2 none = {kNothing, 0.0f}, part = there && own < parts ? a.partial_sums[own * rows + row] : none;
    float top = SHARED ? wave_max(part[0]) : over_lanes<16>(part[0], [](float x, float y) { return fmaxf(x, y); });   // the first 16 threads of a team
    if (SHARED) {
        if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
        __syncthreads();
        top = tops[0];
#pragma unroll
        for (int k = 1; k < kJoinThreads / 64; ++k) top = fmaxf(top, tops[k]);
    }
    float* const mine = weights[SHARED ? 0 : team];
    if (own < parts) mine[own] = Shrink(part[0] - top)(part[1]);
    __syncthreads();
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = SHARED ? team : 0; there && p < parts; p += kStride * kAhead) {
        f32x4 v[kAhead];
        float weight[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = p + k * kStride;
            weight[k] = at < parts ? mine[at] : 0.0f;
            v[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            // a part that saw nothing has written no outputs
            if (!is(weight[k], 0.0f)) v[k] = *reinterpret_cast<const f32x4*>(a.partial + (at * rows + row) * DIM + 4 * column);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(weight[k], v[k][i], sum[i]);
    }
    if (SHARED) {
        sums[team][column] = sum;
        __syncthreads();
        if (team != 0) return;
#pragma unroll
        for (int k = 1; k < kTeams; ++k) sum += sums[k][column];
    }
    if (!there) return;
    float total = 0.0f;
    for (int p = 0; p < parts; ++p) total += mine[p];
    const int64_t token = row / a.q_heads, head = row - token * a.q_heads;
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = is(total, 0.0f) ? 0.0f : sum[i] / total;
    store_some(a.out.p, a.dtype, token * a.out.token + head * a.out.head + 4 * column, f);
}

// ----------------------------------------------------------------------------- launches

constexpr int64_t kMostBlocks = int64_t(1) << 22;
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int ceil_log2(int64_t n) { return n <= 1 ? 0 : 64 - __builtin_clzll(static_cast<unsigned long long>(n - 1)); }

struct Shape {
    int rows;      // of a tile: 16, or 32 per wavefront of the kernel for many rows
    int64_t tiles, parts, per_part;
};

// Which kernel serves, by the rows of a sequence and head of the cache.  The one for few reads and widens the same keys again for every 16 rows, but a
// workgroup of it begins sooner and leaves room for a second; the one for many does so for every 128 or 256.  Few -> many, us, 8 bits, 32 heads over 8:
//   heads of 128       64 rows  one sequence of 8192, bfloat16  24.5 -> 26.9, binary32 32.3 -> 29.6; 16 of 4096  90.7 -> 88.9, 121 -> 130
//                      80 rows                                  28.3 -> 27.9,          37.9 -> 31.3;             120 -> 90.2,  191 -> 130
//                     320 rows                                  46.4 -> 47.6,          77.9 -> 73.0;             264 -> 191,   494 -> 370
//   heads of 64: the workgroups of 16 rows decide, kLoad of them half filling the card
//                     256 rows  one of 8192 (128)               23.1 -> 30.5,          28.2 -> 34.5;   4 of 4096 (512)   32.3 -> 33.6, 41.7 -> 40.8
//                     512 rows               (256)              34.2 -> 37.6,          44.0 -> 43.5             (1024)   57.3 -> 49.4, 76.0 -> 62.6
//                     768 rows               (384)              54.6 -> 44.2,          73.2 -> 54.8;  16 of 4096, 80 rows (640)  66.0 -> 61.4, 71.9 -> 72.5
//   heads of 256, 16-bit types: likewise above 128 rows
//                      80 rows  one of 8192                     59.7 -> 55.4;  4 of 4096  92.0 -> 104;  16 of 4096  408 -> 308
//                     256 rows               (128)              105 -> 121;               (512)  182 -> 175          886 -> 600
//   heads of 256, binary32 (where the many need 600 bytes of scratch memory a lane): the sequences and heads of the cache decide
//                     128 rows  one of 8192 (8)                 124 -> 127;  4 of 4096 (32)  228 -> 253;  16 of 4096 (128)  1027 -> 861
//                    1024 rows                                  611 -> 803;                 1236 -> 1543                    6811 -> 6003
constexpr int64_t kManyRows = 65, kLoad = 256, kManyGroups = 65;

bool many_rows(int32_t dim, bool wide, int64_t groups, int64_t rows)
{
    if (rows < kManyRows) return false;
    const bool loaded = groups * ceil_div(rows, 16) > kLoad;
    return dim == 128 || (dim == 64 ? loaded : wide ? groups >= kManyGroups : rows <= 128 || loaded);
}

// Rows of a workgroup of it: 256 but where they need too many registers, in heads of 256, and for up to 128 rows of binary32 in heads of 128
// (128 -> 256, us: 16 sequences of 4096, 128 rows 137 -> 154, 160 rows 243 -> 169; heads of 64 92 -> 74, bfloat16 in heads of 128 113 -> 94).
int many_rows_of(int32_t dim, bool wide, int64_t rows) { return dim == 256 || (dim == 128 && wide && rows <= 128) ? 128 : 256; }

Shape shape_of(const actq_cache* c, int32_t heads, int64_t sequences, int64_t max_query, int64_t max_length, int32_t window, bool wide)
{
    const int64_t group = heads / c->heads, groups = sequences * c->heads, rows = max_query < 1 ? group : max_query * group;
    Shape s;
    s.rows = many_rows(c->dim, wide, groups, rows) ? many_rows_of(c->dim, wide, rows) : 16;
    s.tiles = ceil_div(rows, s.rows);
    if (s.tiles > kMostBlocks / groups) s.tiles = kMostBlocks / groups;
    // keys of a step; the fewest that are worth a workgroup; workgroups that are wanted, as many as are resident: two per compute unit, one of 256
    // rows.  More of them cost more than they balance (16 rows, 1024 and 2048 instead of 512: 32 sequences of different lengths 85 -> 91, 103 us,
    // one of 32768 23 -> 27, 27)
    const int64_t block = s.rows == 16 ? (c->dim == 256 ? 32 : 64) : 8192 / c->dim;
    const int64_t least = s.rows == 16 ? kFewWaves * block : 256, wanted = s.rows == 256 ? 256 : 512;
    int64_t span = max_length < 1 ? 1 : max_length;
    if (window > 0 && span > window + ceil_div(s.rows, group) + block) span = window + ceil_div(s.rows, group) + block;
    s.parts = wanted / (groups * s.tiles);
    if (s.parts < 1) s.parts = 1;
    if (s.parts > ceil_div(span, least)) s.parts = ceil_div(span, least);
    if (s.parts > kMostParts) s.parts = kMostParts;
    s.per_part = ceil_div(ceil_div(span, s.parts), block) * block;
    s.parts = ceil_div(span, s.per_part);
    return s;
}

// Numbers of binary16 for an element of q and for a weight.  One holds q exactly but for binary32.  A weight of one number costs a bfloat16 result 1 % of its
// error.  A binary16 result it costs up to 70 % where few keys share the weight, so there it has two up to kFewKeys keys: beyond, a key's
// rounding is a small part of a result that does not vanish, and twice the second products cost more (32 sequences of up to 16384, 4 bits
// 81 -> 88 us; 2048 tokens over 32768 1340 -> 1730 us; one token over 1021 0.5 us).
constexpr int64_t kFewKeys = 1024;

template <typename F>
int by_numbers(int dtype, int64_t keys, F f)
{
    constexpr std::integral_constant<int, 1> one;
    constexpr std::integral_constant<int, 2> two;
    return dtype == ACTQ_F32 ? f(two, two) : dtype == ACTQ_F16 && keys <= kFewKeys ? f(one, two) : f(one, one);
}

template <typename F>
int by_bits(int bits, F f)
{
    return bits == 8 ? f(std::integral_constant<int, 8>{}) : f(std::integral_constant<int, 4>{});
}

}  // namespace

uint64_t cache_attention_workspace(const actq_cache* c, int32_t heads, int64_t tokens, int64_t sequences, int64_t max_query, int64_t max_length, int32_t window)
{
    if (tokens == 0 || sequences == 0) return 0;
    int64_t parts = 1;   // of either kind of type: the caller asks without one
    for (const bool wide : {false, true}) {
        const Shape s = shape_of(c, heads, sequences, max_query, max_length, window, wide);
        if (s.parts > parts) parts = s.parts;
    }
    return parts == 1 ? 0 : static_cast<uint64_t>(parts) * tokens * heads * (c->dim + 2) * sizeof(float);
}

int launch_cache_attention(const actq_cache* c, const actq_heads* q, int dtype, int64_t tokens, int64_t sequences, const int32_t* table, int32_t table_width,
                           const int32_t* lengths, const int32_t* query_start, int64_t max_query, int64_t max_length, float scale, float softcap, int32_t window,
                           const actq_heads* out, void* workspace, void* stream)
{
    const char* who = "actq_cache_attention";
    const bool wide = dtype == ACTQ_F32;
    const Shape shape = shape_of(c, q->heads, sequences, max_query, max_length, window, wide);
    AttendArgs a = {};
    a.key_codes = c->key_codes;
    a.key_header = c->key_header;
    a.value_codes = c->value_codes;
    a.value_header = c->value_header;
    a.pages = c->pages;
    a.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
    a.kv_heads = c->heads;
    a.key_bits = c->key_bits;
    a.value_bits = c->value_bits;
    a.q = {q->data, q->token_stride, q->head_stride};
    a.out = {out->data, out->token_stride, out->head_stride};
    a.dtype = dtype;
    a.tokens = static_cast<int32_t>(tokens);
    a.sequences = static_cast<int32_t>(sequences);
    a.q_heads = q->heads;
    a.group = q->heads / c->heads;
    a.by_group = make_fastdiv(static_cast<uint32_t>(a.group));
    a.table = table;
    a.table_width = table_width;
    a.lengths = lengths;
    a.query_start = query_start;
    // A cap beyond 2^60 would overflow in the unit of a row of the smallest elements, and leaves the scores below it as they are; one below 2^-60 would
    // in its inverse, and leaves all weights alike.
    const float cap = softcap > kMostCap ? kMostCap : softcap > 0.0f && softcap < kLeastCap ? kLeastCap : softcap;
    a.factor = cap > 0.0f ? scale / cap : scale * kLog2e;
    a.cap = cap * kLog2e;
    a.window = window;
    // p <= 2^(kMostWeight - least), and there are no more of them than the table has room for
    a.least = static_cast<float>(ceil_log2(static_cast<int64_t>(table_width) << a.page_shift) - 111);
    a.tiles = static_cast<uint32_t>(shape.tiles);
    a.parts = static_cast<uint32_t>(shape.parts);
    a.by_tiles = make_fastdiv(a.tiles);
    a.by_parts = make_fastdiv(a.parts);
    a.by_heads = make_fastdiv(static_cast<uint32_t>(c->heads));
    a.per_part = static_cast<int32_t>(shape.per_part);
    if (shape.parts > 1) {
        a.partial = static_cast<float*>(workspace);
        a.partial_sums = reinterpret_cast<f32x2*>(a.partial + shape.parts * tokens * q->heads * c->dim);
    }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned blocks = static_cast<unsigned>(sequences * c->heads * shape.parts * shape.tiles);
    const int rc = by_dim(c->dim, [&](auto d) {
        return by_numbers(dtype, window > 0 && window < max_length ? window : max_length, [&](auto split, auto weights) {
            constexpr int kDim = decltype(d)::value, kSplit = decltype(split)::value, kWeights = decltype(weights)::value;
            if (shape.rows == 256) {
                if constexpr (kDim != 256) launch(attend_many_kernel<kDim, kSplit, kWeights, 8>, blocks, 512, s, a);
                return launched(who);
            }
            if (shape.rows == 128) {
                if constexpr (kDim == 256 || (kDim == 128 && kSplit == 2)) launch(attend_many_kernel<kDim, kSplit, kWeights, 4>, blocks, 256, s, a);
                return launched(who);
            }
            return by_bits(c->key_bits, [&](auto kb) {
                return by_bits(c->value_bits, [&](auto vb) {
                    launch(attend_few_kernel<kDim, kSplit, kWeights, decltype(kb)::value, decltype(vb)::value>, blocks, kFewWaves * 64, s, a);
                    return launched(who);
                });
            });
        });
    });
    if (rc != ACTQ_OK || shape.parts == 1) return rc;
    return by_dim(c->dim, [&](auto d) {
        constexpr int kDim = decltype(d)::value;
        const int64_t rows = tokens * q->heads;
        if (shape.parts >= kSharedParts) launch(attend_join_kernel<kDim, true>, static_cast<unsigned>(rows), kJoinThreads, s, a);
        else launch(attend_join_kernel<kDim, false>, static_cast<unsigned>(ceil_div(rows, kJoinThreads / (kDim / 4))), kJoinThreads, s, a);
        return launched(who);
    });
}

}  // namespace actq
