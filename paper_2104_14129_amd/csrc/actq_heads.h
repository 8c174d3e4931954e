// What the kernels for attention heads share: tensors of heads, eight neighbouring elements of a head per lane, sums over the lanes of a head,
// the rotation by position, the quantizer of the cache.
#ifndef ACTQ_HEADS_H
#define ACTQ_HEADS_H

#include <cstdint>
#include <type_traits>

#include <hip/hip_runtime.h>

#include "actq_internal.h"

namespace actq {

constexpr int kLaneValues = 8;   // elements of a head that a lane holds: 16 bytes of a 16-bit type; 8, 16 or 32 lanes hold a head of 64, 128 or 256

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Element types: binary32, binary16 and bfloat16 (as __bf16, whose conversions round to nearest, ties to even).
template <typename F>
inline int by_dtype(int dt, F f)
{
    return dt == ACTQ_F32 ? f(float{}) : dt == ACTQ_F16 ? f(_Float16{}) : f(__bf16{});
}

template <typename F>
inline int by_dim(int dim, F f)
{
    return dim == 64 ? f(std::integral_constant<int, 64>{}) : dim == 128 ? f(std::integral_constant<int, 128>{}) : f(std::integral_constant<int, 256>{});
}

// Eight neighbouring elements as loaded, and as binary32.  A tensor is aligned to its element size only: global
// accesses of any width may start at any byte.
template <typename T>
struct Eight {
    typedef T vector __attribute__((ext_vector_type(8)));
    typedef vector unaligned __attribute__((aligned(sizeof(T))));
    vector v;

    __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const unaligned*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<unaligned*>(p) = v; }
    __device__ __forceinline__ void widen(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(v[i]);
    }
    __device__ __forceinline__ void round(const float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<T>(f[i]);
    }
};

// The bits of a value that may be no number.  The compiler takes it that floating-point data holds no NaN, and would fold a
// question about the bits that it recognises as one about the number.
__device__ __forceinline__ uint32_t bits_of(float v)
{
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    asm("" : "+v"(b));
    return b;
}

// The magnitude of a value as a whole number, which orders infinities and NaN above all numbers.
__device__ __forceinline__ uint32_t magnitude(float v) { return bits_of(v) & 0x7fffffffu; }

__device__ __forceinline__ float nan_where(bool bad)
{
    uint32_t b = bad ? 0x7fc00000u : 0u;
    asm("" : "+v"(b));
    return __builtin_bit_cast(float, b);
}

// A value of another lane of the 16-lane row, by a DPP control: every lane has a source, so that the instruction which
// uses the value can fetch it itself.
template <int CONTROL>
__device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
}

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140, kDppBroadcast = 0x150;

// sum + v of lane AT of the 16-lane row * factor, in one instruction; the compiler makes two of it (2048 tokens over 32768 1334 -> 1628 us).
// Of an instruction of ours it does not know what it has to wait for: a value that has just been written takes two cycles to be seen
// by other lanes, so `settled` goes first; and the result of an exponential one cycle to be seen at all, so `after` is something that was
// computed from it.  That nothing has come between is looked up in the assembly of every build, which fails otherwise: eight of them behind a wait in
// one block of assembly would need no such check, but cost the schedule nearly as much (1573 us); a wait in each costs less (1452 us).
__device__ __forceinline__ void settled(float& v) { asm volatile("s_nop 1" : "+v"(v)); }

template <int AT>
__device__ __forceinline__ float add_broadcast(float sum, float v, float factor, float after)
{
    asm("v_fmac_f32_dpp %0, %1, %2 row_newbcast:%3 row_mask:0xf bank_mask:0xf" : "+v"(sum) : "v"(v), "v"(factor), "n"(AT), "v"(after));
    return sum;
}

// op over the LANES lanes of a head, in all of them: neighbours, pairs, then mirrored halves, whose lanes are alike by then.
template <int LANES, typename Op>
__device__ __forceinline__ float over_lanes(float v, Op op)
{
    v = op(v, dpp<kDppXor1>(v));
    v = op(v, dpp<kDppXor2>(v));
    v = op(v, dpp<kDppHalfMirror>(v));
    if (LANES >= 16) v = op(v, dpp<kDppMirror>(v));
    if (LANES >= 32) v = op(v, __shfl_xor(v, 16));
    if (LANES >= 64) v = op(v, __shfl_xor(v, 32));
    return v;
}

template <int LANES>
__device__ __forceinline__ float sum_over_lanes(float v)
{
    return over_lanes<LANES>(v, [](float a, float b) { return a + b; });
}

// A tensor [tokens, heads, dim] whose heads are contiguous.
template <typename T>
struct HeadsOf {
    T* p;
    int64_t token, head;   // strides in elements
};

template <typename T>
inline HeadsOf<T> heads_of(const actq_heads* h)
{
    if (!h) return {nullptr, 0, 0};
    return {static_cast<T*>(h->data), h->token_stride, h->head_stride};
}

struct Rotation {
    const int32_t* positions;
    const float* cos;
    const float* sin;
    int64_t rows;
    int32_t half;          // pairs per head
    int32_t interleaved;   // pairs (2p, 2p + 1) instead of (p, p + half)
};

struct Weights {
    const void* q;   // null: ones
    const void* k;
    int32_t wide;    // binary32 beside a 16-bit type of the heads
};

// The lane's part of the rotation of one token.
template <int LANES>
struct Turn {
    float c[8], s[8];
    bool turned;   // whether the lane's elements are rotated
    int partner;   // lane that holds the other elements of the pairs

    // A lane's place among the LANES of its head.
    __device__ __forceinline__ void load(const Rotation& r, int64_t position, int lane)
    {
        const int at = lane % LANES, first = kLaneValues * at;
        turned = first < 2 * r.half;
        partner = lane;
        if (!turned) return;
        if (r.interleaved) {
            const float* const cs = r.cos + position * r.half + first / 2;
            const float* const sn = r.sin + position * r.half + first / 2;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[2 * i] = c[2 * i + 1] = cs[i];
                s[2 * i] = -sn[i];
                s[2 * i + 1] = sn[i];
            }
        } else {
            const bool low = first < r.half;
            const int64_t entry = position * r.half + (low ? first : first - r.half);
            partner = low ? lane + r.half / kLaneValues : lane - r.half / kLaneValues;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = r.cos[entry + i];
                const float sn = r.sin[entry + i];
                s[i] = low ? -sn : sn;
            }
        }
    }

    // v rotated; BACK: by the opposite angle.
    template <bool BACK>
    __device__ __forceinline__ void apply(float (&v)[8], int interleaved) const
    {
        float other[8];
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = v[i ^ 1];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = __shfl(v[i], partner);
        }
        if (!turned) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(BACK ? -s[i] : s[i], other[i], v[i] * c[i]);
    }
};

template <typename T>
__device__ __forceinline__ void load_weight(const void* w, int wide, int first, float (&f)[8])
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 1.0f;
    } else if (wide) {
        Eight<float> e;
        e.load(static_cast<const float*>(w) + first);
        e.widen(f);
    } else {
        Eight<T> e;
        e.load(static_cast<const T*>(w) + first);
        e.widen(f);
    }
}

inline Rotation rotation_of(const actq_rotation* r)
{
    return {r->positions, r->cos, r->sin, r->rows, r->rotated / 2, r->interleaved};
}

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

// A launch has fewer than 2^32 threads: what needs more goes in several, f(first, blocks) each.
template <typename F>
inline void launches(int64_t blocks, int threads, F f)
{
    const int64_t most = ((int64_t(1) << 32) - 1) / threads;
    for (int64_t first = 0; first < blocks; first += most) f(first, static_cast<unsigned>(blocks - first < most ? blocks - first : most));
}

inline int launched(const char* who)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(ACTQ_EHIP, "%s: launch failed: %s", who, hipGetErrorString(e));
    return ACTQ_OK;
}

}  // namespace actq

#endif
