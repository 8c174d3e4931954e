// New tokens on their way into a paged cache: queries and keys normed (or not) and rotated by position, keys and values quantised into
// their slots, in one launch.
//
//   n = x r w,  r = (mean(x^2) + eps)^(-1/2), or n = x;  y = n rotated by the token's position
//   queries: y is stored;  keys: y, values: x go as groups into the cache
//
// What bounds it: memory, and for one token of each sequence the launch.  Beside the norm and the write as two calls, the keys are neither written
// and read once more nor rounded to their type between.  A code changes where its value passes a border between two, so a key's codes would go by the
// order of the sums in its norm: keys are computed in binary64, up to the one rounding to binary32 that the codes are defined on.  That is 30 operations
// for each of a key's elements.
//
// Measured on one MI355X, whose copy of 1 GiB reaches 5.1 TB/s: 8191 tokens of 32 heads over 8 of 128 in binary16, to 4 bits, 45 us (4.0 TB/s; with three wavefronts a SIMD
// instead of four 50), 32 tokens 5.1 us; the same tokens in binary32 76 us (4.5 TB/s).  Norm and write as two calls, from the host on the same inputs again and again: 9.1 us instead of 5.0
// for the 32 tokens, 40.9 instead of 39.3 for the 8191, where the binary64 of the keys costs about what the round trip saves.
#include "actq_heads.h"

namespace actq {
namespace {

constexpr int kAppendWaves = 4;
constexpr int kAppendBlock = kAppendWaves * 64;

template <typename T>
struct AppendArgs {
    HeadsOf<T> q, k, v, q_out;
    uint8_t* key_codes;
    float* key_header;
    uint8_t* value_codes;
    float* value_header;
    const int64_t* slots;
    int64_t slot_count;
    int32_t q_heads, heads;        // of the queries, of keys and values
    int32_t q_steps, all_steps;    // steps of 64 / LANES heads: of the queries, then as many of the keys as of the values
    int32_t page_shift, key_bits, value_bits;
    int32_t norm;
    int64_t tokens;
    uint32_t parts, per_part;      // wavefronts of a token, steps of each
    FastDiv by_parts;
    Rotation rotation;
    Weights weights;
    float eps;
};

template <int LANES>
__device__ __forceinline__ double double_sum_over_lanes(double v)
{
#pragma unroll
    for (int step = 1; step < LANES; step *= 2) v += __shfl_xor(v, step);
    return v;
}

// A key in binary64, rounded to binary32.
template <int LANES>
__device__ __forceinline__ void exact_key(float (&x)[8], const float (&w)[8], const Turn<LANES>& turn, bool norm, float eps, int interleaved)
{
    double n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] = static_cast<double>(x[i]);
    if (norm) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma(n[i], n[i], sum);
        sum = double_sum_over_lanes<LANES>(sum);
        const double r = 1.0 / sqrt(sum * (1.0 / (LANES * kLaneValues)) + static_cast<double>(eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) n[i] = n[i] * r * static_cast<double>(w[i]);
    }
    double other[8];
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = n[i ^ 1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl(n[i], turn.partner);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (turn.turned) n[i] = fma(static_cast<double>(turn.s[i]), other[i], n[i] * static_cast<double>(turn.c[i]));
        x[i] = static_cast<float>(n[i]);
    }
}

// Heads in flight per lane.
constexpr int kAhead = 4;

template <typename T, int LANES>
__global__ __launch_bounds__(kAppendBlock, 4) void cache_append_kernel(AppendArgs<T> a)
{
    constexpr int kSide = 64 / LANES, kDim = LANES * kLaneValues;
    const int lane = threadIdx.x % 64, at = lane % LANES, first = kLaneValues * at, side = lane / LANES;
    const uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * kAppendWaves + threadIdx.x / 64);
    const uint32_t token = (__umulhi(unit, a.by_parts.m) + unit) >> a.by_parts.s;
    if (token >= a.tokens) return;
    const int begin = (unit - token * a.parts) * a.per_part, end = min(begin + static_cast<int>(a.per_part), a.all_steps);
    const int64_t position = a.rotation.positions[token], slot = a.slots[token];
    const bool padding = position < 0 || position >= a.rotation.rows, held = slot >= 0 && slot < a.slot_count;
    const int64_t page = slot >> a.page_shift, offset = slot - (page << a.page_shift);
    const int k_steps = (a.all_steps - a.q_steps) / 2, v_begin = a.q_steps + k_steps;
    Turn<LANES> turn;
    turn.load(a.rotation, padding ? 0 : position, lane);
    float qw[8], kw[8];
    load_weight<T>(a.weights.q, a.weights.wide, first, qw);
    load_weight<T>(a.weights.k, a.weights.wide, first, kw);
    for (int from = begin; from < end; from += kAhead) {
        Eight<T> in[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int step = from + u;
            const HeadsOf<T>& x = step < a.q_steps ? a.q : step < v_begin ? a.k : a.v;
            const int head = (step < a.q_steps ? step : step < v_begin ? step - a.q_steps : step - v_begin) * kSide + side;
            in[u].v = {};
            if (step < end && head < (step < a.q_steps ? a.q_heads : a.heads)) in[u].load(x.p + token * x.token + head * x.head + first);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int step = from + u;
            if (step >= end) break;
            float x[8];
            in[u].widen(x);
            if (step < a.q_steps) {
                const int head = step * kSide + side;
                if (a.norm) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
                    sum = sum_over_lanes<LANES>(sum);
                    const float r = 1.0f / sqrtf(fmaf(sum, 1.0f / kDim, a.eps));
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * qw[i];
                }
                turn.template apply<false>(x, a.rotation.interleaved);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = padding ? 0.0f : x[i];
                in[u].round(x);
                if (head < a.q_heads) in[u].store(a.q_out.p + token * a.q_out.token + head * a.q_out.head + first);
                continue;
            }
            const bool of_v = step >= v_begin;
            const int head = (of_v ? step - v_begin : step - a.q_steps) * kSide + side;
            const int64_t row = ((page * a.heads + head) << a.page_shift) + offset;
            const bool there = held && head < a.heads;
            if (of_v) {
                quantise<LANES>(x, a.value_bits, a.value_codes + row * (kDim / 8 * a.value_bits), a.value_header + 2 * row, there, at);
            } else {
                exact_key<LANES>(x, kw, turn, a.norm, a.eps, a.rotation.interleaved);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = padding ? 0.0f : x[i];
                quantise<LANES>(x, a.key_bits, a.key_codes + row * (kDim / 8 * a.key_bits), a.key_header + 2 * row, there, at);
            }
        }
    }
}

// Wavefronts that a pass is cut into where there are few tokens: 16 per compute unit, as in the norm of heads.
constexpr int64_t kAppendUnits = 4096;

}  // namespace

int launch_cache_append(const actq_cache* c, const actq_heads* q, const actq_heads* k, const actq_heads* v, int dtype, int64_t tokens, const void* q_weight,
                        const void* k_weight, int weight_dtype, const actq_rotation* rotation, int norm, float eps, const int64_t* slots, const actq_heads* q_out, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        return by_dim(c->dim, [&](auto d) {
            typedef decltype(type) T;
            constexpr int kLanes = decltype(d)::value / kLaneValues, kSide = 64 / kLanes;
            AppendArgs<T> a = {};
            a.q = heads_of<T>(q);
            a.k = heads_of<T>(k);
            a.v = heads_of<T>(v);
            a.q_out = heads_of<T>(q_out);
            a.key_codes = c->key_codes;
            a.key_header = c->key_header;
            a.value_codes = c->value_codes;
            a.value_header = c->value_header;
            a.slots = slots;
            a.slot_count = c->pages * c->page_size;
            a.q_heads = q ? q->heads : 0;
            a.heads = c->heads;
            a.q_steps = (a.q_heads + kSide - 1) / kSide;
            a.all_steps = a.q_steps + 2 * ((a.heads + kSide - 1) / kSide);
            a.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
            a.key_bits = c->key_bits;
            a.value_bits = c->value_bits;
            a.norm = norm;
            a.tokens = tokens;
            const int64_t parts = kAppendUnits / tokens < 1 ? 1 : kAppendUnits / tokens < a.all_steps ? kAppendUnits / tokens : a.all_steps;
            a.per_part = static_cast<uint32_t>((a.all_steps + parts - 1) / parts);
            a.parts = (a.all_steps + a.per_part - 1) / a.per_part;
            a.by_parts = make_fastdiv(a.parts);
            a.rotation = rotation_of(rotation);
            a.weights = {q_weight, k_weight, weight_dtype == ACTQ_F32};
            a.eps = eps;
            const uint64_t units = static_cast<uint64_t>(tokens) * a.parts;
            launch(cache_append_kernel<T, kLanes>, static_cast<unsigned>((units + kAppendWaves - 1) / kAppendWaves), kAppendBlock, static_cast<hipStream_t>(stream), a);
            return launched("actq_cache_append");
        });
    });
}

}  // namespace actq
