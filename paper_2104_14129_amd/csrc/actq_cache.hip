// A paged cache of keys and values, quantised as it is written, and read back.
//
// A group is a token's head: Z = min, R = max - min, code = nearest((x - Z) (B / R)), ties to even, B = 2^bits - 1, and a code
// stands for Z + code (R / B); a group with an infinity or NaN, or whose R overflows, reads as NaN.  It is the codec's quantizer with
// rounding to nearest in place of the stochastic one, since a cache feeds no gradient that would have to be unbiased, and to nearest is
// half the error.
//
// What bounds it: memory.  A head is 8, 16 or 32 lanes of eight elements; a lane handles a token's key and value together, so that
// the slot is looked up once and two loads are in flight.  Measured on one MI355X, whose copy of 1 GiB reaches 5.2 TB/s: 65536 tokens of 8 heads of 128
// read from 8 bits to bfloat16 83 us (5.0 TB/s), 8191 tokens written from binary16 to 4 bits 12.9 us (3.3 TB/s), 64 tokens 3 us.
#include "actq_heads.h"

namespace actq {
namespace {

constexpr int kCacheBlock = 256;

template <typename T>
struct CacheArgs {
    HeadsOf<T> k, v;
    uint8_t* key_codes;      // [pages, heads, page_size, dim * bits / 8]
    float* key_header;       // [pages, heads, page_size, 2]
    uint8_t* value_codes;
    float* value_header;
    const int64_t* slots;
    int64_t slot_count;      // pages * page_size
    int32_t heads, page_shift;
    uint32_t units;          // tokens * heads
    FastDiv by_heads;
    int32_t key_bits, value_bits;
};

// The unit of a thread: a token's head.
template <typename T>
struct Unit {
    uint32_t token, head;
    int64_t row;     // of the head's token in the pages
    bool there;      // false beyond the last unit
    bool held;       // whether the slot is one of the cache's

    __device__ __forceinline__ Unit(const CacheArgs<T>& a, uint32_t unit)
    {
        there = unit < a.units;
        const uint32_t u = there ? unit : 0;
        token = (__umulhi(u, a.by_heads.m) + u) >> a.by_heads.s;
        head = u - token * a.heads;
        const int64_t slot = a.slots[token];
        held = there && slot >= 0 && slot < a.slot_count;
        const int64_t page = slot >> a.page_shift, offset = slot - (page << a.page_shift);
        row = ((page * a.heads + head) << a.page_shift) + offset;
    }
};

// Codes of a lane's eight elements into the stream, the group's header by its first lane.
template <int LANES>
__device__ __forceinline__ void quantise(const float (&x)[8], int bits, uint8_t* codes, float* header, bool held, int at)
{
    float low = x[0], high = x[0];
    uint32_t largest = magnitude(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
        largest = max(largest, magnitude(x[i]));
    }
    // an infinity or NaN (which a minimum passes over) gives the group an infinite range
    if (largest >= 0x7f800000u) {
        low = 0.0f;
        high = INFINITY;
    }
    low = over_lanes<LANES>(low, [](float a, float b) { return fminf(a, b); });
    high = over_lanes<LANES>(high, [](float a, float b) { return fmaxf(a, b); });
    const float top = bits == 8 ? 255.0f : 15.0f;
    const float zero = low + 0.0f;   // -0 becomes +0
    const float range = high - zero;
    const bool none = magnitude(range) >= 0x7f800000u;
    float inverse = top / range, step = range / top;
    if (range == 0.0f || isinf(inverse)) inverse = step = 0.0f;
    uint32_t code[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) code[i] = none ? 0u : static_cast<uint32_t>(rintf(fminf((x[i] - zero) * inverse, top)));
    if (!held) return;
    if (bits == 8) {
        u32x2 w;
        w[0] = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
        w[1] = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
        *reinterpret_cast<u32x2*>(codes + 8 * at) = w;
    } else {
        uint32_t w = code[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) w |= code[i] << 4 * i;
        *reinterpret_cast<uint32_t*>(codes + 4 * at) = w;
    }
    if (at == 0) {
        const uint32_t nan = 0x7fc00000u;   // stored as bits: the compiler takes it that floating-point data holds no NaN
        *reinterpret_cast<u32x2*>(header) = none ? u32x2{nan, nan} : u32x2{__builtin_bit_cast(uint32_t, zero), __builtin_bit_cast(uint32_t, step)};
    }
}

template <typename T, int LANES>
__global__ __launch_bounds__(kCacheBlock) void cache_write_kernel(CacheArgs<T> a)
{
    constexpr int kDim = LANES * kLaneValues;
    const int at = threadIdx.x % LANES;
    const Unit<T> u(a, blockIdx.x * (kCacheBlock / LANES) + threadIdx.x / LANES);
    Eight<T> ek, ev;
    ek.load(a.k.p + u.token * a.k.token + u.head * a.k.head + kLaneValues * at);
    ev.load(a.v.p + u.token * a.v.token + u.head * a.v.head + kLaneValues * at);
    float x[8];
    ek.widen(x);
    quantise<LANES>(x, a.key_bits, a.key_codes + u.row * (kDim / 8 * a.key_bits), a.key_header + 2 * u.row, u.held, at);
    ev.widen(x);
    quantise<LANES>(x, a.value_bits, a.value_codes + u.row * (kDim / 8 * a.value_bits), a.value_header + 2 * u.row, u.held, at);
}

// A lane's eight codes as loaded; of 4 bits in the first word.
__device__ __forceinline__ u32x2 load_codes(const uint8_t* codes, int bits, int at)
{
    if (bits == 8) return *reinterpret_cast<const u32x2*>(codes + 8 * at);
    return u32x2{*reinterpret_cast<const uint32_t*>(codes + 4 * at), 0u};
}

__device__ __forceinline__ void dequantise(u32x2 w, int bits, f32x2 header, float (&x)[8])
{
    if (bits == 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(static_cast<float>(w[i / 4] >> 8 * (i % 4) & 255u), header[1], header[0]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(static_cast<float>(w[0] >> 4 * i & 15u), header[1], header[0]);
    }
}

template <typename T, int LANES>
__global__ __launch_bounds__(kCacheBlock) void cache_read_kernel(CacheArgs<T> a)
{
    constexpr int kDim = LANES * kLaneValues;
    const int at = threadIdx.x % LANES;
    const Unit<T> u(a, blockIdx.x * (kCacheBlock / LANES) + threadIdx.x / LANES);
    if (!u.there) return;
    u32x2 wk = {}, wv = {};
    f32x2 hk = {}, hv = {};   // a slot that is none reads as zeros
    if (u.held) {
        wk = load_codes(a.key_codes + u.row * (kDim / 8 * a.key_bits), a.key_bits, at);
        wv = load_codes(a.value_codes + u.row * (kDim / 8 * a.value_bits), a.value_bits, at);
        hk = *reinterpret_cast<const f32x2*>(a.key_header + 2 * u.row);
        hv = *reinterpret_cast<const f32x2*>(a.value_header + 2 * u.row);
    }
    float x[8];
    Eight<T> e;
    dequantise(wk, a.key_bits, hk, x);
    e.round(x);
    e.store(a.k.p + u.token * a.k.token + u.head * a.k.head + kLaneValues * at);
    dequantise(wv, a.value_bits, hv, x);
    e.round(x);
    e.store(a.v.p + u.token * a.v.token + u.head * a.v.head + kLaneValues * at);
}

template <typename T>
CacheArgs<T> cache_args(const actq_cache* c, const actq_heads* k, const actq_heads* v, int64_t tokens, const int64_t* slots)
{
    CacheArgs<T> a = {};
    a.k = heads_of<T>(k);
    a.v = heads_of<T>(v);
    a.key_codes = c->key_codes;
    a.key_header = c->key_header;
    a.value_codes = c->value_codes;
    a.value_header = c->value_header;
    a.slots = slots;
    a.slot_count = c->pages * c->page_size;
    a.heads = c->heads;
    a.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
    a.units = static_cast<uint32_t>(tokens * c->heads);
    a.by_heads = make_fastdiv(static_cast<uint32_t>(c->heads));
    a.key_bits = c->key_bits;
    a.value_bits = c->value_bits;
    return a;
}

}  // namespace

int launch_cache_write(const actq_cache* c, const actq_heads* k, const actq_heads* v, int dtype, int64_t tokens, const int64_t* slots, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        return by_dim(c->dim, [&](auto d) {
            typedef decltype(type) T;
            constexpr int kLanes = decltype(d)::value / kLaneValues, kUnits = kCacheBlock / kLanes;
            const CacheArgs<T> a = cache_args<T>(c, k, v, tokens, slots);
            launch(cache_write_kernel<T, kLanes>, (a.units + kUnits - 1) / kUnits, kCacheBlock, static_cast<hipStream_t>(stream), a);
            return launched("actq_cache_write");
        });
    });
}

int launch_cache_read(const actq_cache* c, const actq_heads* k, const actq_heads* v, int dtype, int64_t tokens, const int64_t* slots, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        return by_dim(c->dim, [&](auto d) {
            typedef decltype(type) T;
            constexpr int kLanes = decltype(d)::value / kLaneValues, kUnits = kCacheBlock / kLanes;
            const CacheArgs<T> a = cache_args<T>(c, k, v, tokens, slots);
            launch(cache_read_kernel<T, kLanes>, (a.units + kUnits - 1) / kUnits, kCacheBlock, static_cast<hipStream_t>(stream), a);
            return launched("actq_cache_read");
        });
    });
}

}  // namespace actq
