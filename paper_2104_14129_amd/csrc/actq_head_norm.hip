// RMS norm of every query and key head with the rotation by position in the same pass, and its gradient.
//
//   n = x r w,  r = (mean(x^2) + eps)^(-1/2)           over the `dim` elements of a head
//   y_i = n_i c - n_j s,  y_j = n_j c + n_i s          for the pairs (i, j) of the first `rotated` elements
// and with g the gradient of n (that of y rotated back):
//   grad_x = r (g w - x r^2 mean(g w x)),  grad_w = sum over tokens and heads of g x r
//
// What bounds it: memory.  A pass reads and writes every head once (backward: reads two, writes one).  A wavefront takes one
// token and holds what its heads share (cosines, sines, weights) in registers, 8, 4 or 2 heads side by side at 8, 16 or 32 lanes,
// so that the tables are read once per token and not once per head.  The partner of an element sits rotated / 2 elements
// away in another lane and comes by a lane exchange.  All arithmetic is binary32; a result is rounded once.
//
// Measured on one MI355X, whose copy of 1 GiB reaches 5.2 TB/s: 8192 tokens of 32 + 8 heads of 128 in binary16 30 us (5.8 TB/s), eight tokens
// 3.7 us; gradients of 16384 such tokens in bfloat16 101 + 5 us (5.1 TB/s), of 4095 tokens of 12 + 4 heads of 64 in binary32 15 + 4 us (3.5 TB/s:
// two tokens per wavefront, one behind the other).
#include "actq_heads.h"

namespace actq {
namespace {

constexpr int kNormWaves = 4;
constexpr int kNormBlock = kNormWaves * 64;

// The steps of a token: groups of 64 / LANES heads of the queries, then of the keys.
struct Steps {
    int32_t q_heads, k_heads;
    int32_t q, all;     // steps of the queries, of both
};

template <typename T>
struct NormArgs {
    HeadsOf<T> q, k, q_out, k_out;
    Steps steps;
    int64_t tokens;
    uint32_t parts, per_part;   // wavefronts of a token, steps of each
    FastDiv by_parts;
    Rotation rotation;
    Weights weights;
    float eps;
};

// Heads in flight per lane [1: latency shows; 4: what 40 heads need].
constexpr int kAhead = 4;

template <typename T, int LANES>
__global__ __launch_bounds__(kNormBlock) void head_norm_kernel(NormArgs<T> a)
{
    constexpr int kSide = 64 / LANES;   // heads side by side
    const int lane = threadIdx.x % 64, first = kLaneValues * (lane % LANES), side = lane / LANES;
    const uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * kNormWaves + threadIdx.x / 64);
    const uint32_t token = (__umulhi(unit, a.by_parts.m) + unit) >> a.by_parts.s;
    if (token >= a.tokens) return;
    const int begin = (unit - token * a.parts) * a.per_part, end = min(begin + static_cast<int>(a.per_part), a.steps.all);
    const int64_t position = a.rotation.positions[token];
    const bool padding = position < 0 || position >= a.rotation.rows;
    Turn<LANES> turn;
    turn.load(a.rotation, padding ? 0 : position, lane);
    float qw[8], kw[8];
    load_weight<T>(a.weights.q, a.weights.wide, first, qw);
    load_weight<T>(a.weights.k, a.weights.wide, first, kw);
    for (int at = begin; at < end; at += kAhead) {
        Eight<T> in[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int step = at + u;
            const bool of_k = step >= a.steps.q;
            const int head = (of_k ? step - a.steps.q : step) * kSide + side;
            const HeadsOf<T>& x = of_k ? a.k : a.q;
            in[u].v = {};
            if (step < end && head < (of_k ? a.steps.k_heads : a.steps.q_heads)) in[u].load(x.p + token * x.token + head * x.head + first);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int step = at + u;
            if (step >= end) break;
            const bool of_k = step >= a.steps.q;
            const int head = (of_k ? step - a.steps.q : step) * kSide + side;
            const HeadsOf<T>& y = of_k ? a.k_out : a.q_out;
            float v[8], sum = 0.0f;
            in[u].widen(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(v[i], v[i], sum);
            sum = sum_over_lanes<LANES>(sum);
            const float r = 1.0f / sqrtf(fmaf(sum, 1.0f / (LANES * kLaneValues), a.eps));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] * r * (of_k ? kw[i] : qw[i]);
            turn.template apply<false>(v, a.rotation.interleaved);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = padding ? 0.0f : v[i];
            in[u].round(v);
            if (head < (of_k ? a.steps.k_heads : a.steps.q_heads)) in[u].store(y.p + token * y.token + head * y.head + first);
        }
    }
}

template <typename T>
struct NormGradArgs {
    HeadsOf<T> gq, gk, q, k, q_out, k_out;   // gradients of the outputs, inputs, gradients of the inputs
    Steps steps;
    int64_t tokens;
    Rotation rotation;
    Weights weights;
    float eps;
    float* partial;   // [workgroups][queries, keys][dim]; null: no gradient of the weights
};

// Every wavefront goes through the tokens with the grid's stride and keeps its share of both weights' gradients in registers; a
// workgroup's wavefronts join theirs in the LDS in a fixed order.
template <typename T, int LANES>
__global__ __launch_bounds__(kNormBlock) void head_norm_backward_kernel(NormGradArgs<T> a)
{
    constexpr int kSide = 64 / LANES, kDim = LANES * kLaneValues, kPair = 2;
    __shared__ float joined[kNormWaves][2][kDim];
    const int lane = threadIdx.x % 64, first = kLaneValues * (lane % LANES), side = lane / LANES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    float w[2][8], grad_w[2][8];
    load_weight<T>(a.weights.q, a.weights.wide, first, w[0]);
    load_weight<T>(a.weights.k, a.weights.wide, first, w[1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) grad_w[0][i] = grad_w[1][i] = 0.0f;
    for (int64_t token = static_cast<int64_t>(blockIdx.x) * kNormWaves + wave; token < a.tokens; token += static_cast<int64_t>(gridDim.x) * kNormWaves) {
        const int64_t position = a.rotation.positions[token];
        const bool padding = position < 0 || position >= a.rotation.rows;
        Turn<LANES> turn;
        turn.load(a.rotation, padding ? 0 : position, lane);
        const auto pass = [&](const HeadsOf<T>& gy, const HeadsOf<T>& in, const HeadsOf<T>& out, int heads, const float (&weight)[8], float (&sum_w)[8]) {
            for (int at = 0; at < heads; at += kPair * kSide) {
                Eight<T> eg[kPair], ex[kPair];
#pragma unroll
                for (int u = 0; u < kPair; ++u) {
                    const int head = at + u * kSide + side;
                    eg[u].v = {};
                    ex[u].v = {};
                    if (head < heads && !padding) {
                        eg[u].load(gy.p + token * gy.token + head * gy.head + first);
                        ex[u].load(in.p + token * in.token + head * in.head + first);
                    }
                }
#pragma unroll
                for (int u = 0; u < kPair; ++u) {
                    const int head = at + u * kSide + side;
                    float g[8], x[8], square = 0.0f, along = 0.0f;
                    eg[u].widen(g);
                    ex[u].widen(x);
                    turn.template apply<true>(g, a.rotation.interleaved);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        square = fmaf(x[i], x[i], square);
                        along = fmaf(g[i] * weight[i], x[i], along);
                    }
                    square = sum_over_lanes<LANES>(square);
                    along = sum_over_lanes<LANES>(along);
                    const float r = 1.0f / sqrtf(fmaf(square, 1.0f / kDim, a.eps));
                    const float back = along * (1.0f / kDim) * r * r;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sum_w[i] = fmaf(g[i], x[i] * r, sum_w[i]);
                        g[i] = r * fmaf(-x[i], back, g[i] * weight[i]);
                    }
                    eg[u].round(g);
                    if (head < heads) eg[u].store(out.p + token * out.token + head * out.head + first);
                }
            }
        };
        pass(a.gq, a.q, a.q_out, a.steps.q_heads, w[0], grad_w[0]);
        pass(a.gk, a.k, a.k_out, a.steps.k_heads, w[1], grad_w[1]);
    }
    if (!a.partial) return;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = grad_w[which][i];
#pragma unroll
            for (int step = LANES; step < 64; step *= 2) v += __shfl_xor(v, step);
            if (side == 0) joined[wave][which][first + i] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kDim; i += kNormBlock) {
        const float* const at = &joined[0][0][0] + i;
        a.partial[static_cast<int64_t>(blockIdx.x) * 2 * kDim + i] = (at[0] + at[2 * kDim]) + (at[4 * kDim] + at[6 * kDim]);
    }
}

// grad_w [dim] of the queries and of the keys: the workgroups' shares in binary64, each of 64 threads a 64th of them.
constexpr int kSumColumns = 16, kSumRows = 64, kSumAhead = 8;

template <typename W>
__global__ __launch_bounds__(kSumColumns* kSumRows) void head_norm_weights_kernel(const float* partial, int32_t blocks, int32_t dim, W* grad_q, W* grad_k)
{
    __shared__ double sums[kSumRows][kSumColumns];
    const int column = threadIdx.x % kSumColumns, row = threadIdx.x / kSumColumns, at = blockIdx.x * kSumColumns + column;
    double sum = 0.0;
    // all of a thread's loads in flight: one after the other each costs a trip to memory
    for (int b = row; b < blocks; b += kSumRows * kSumAhead) {
        float v[kSumAhead];
#pragma unroll
        for (int k = 0; k < kSumAhead; ++k) {
            const int from = b + k * kSumRows;
            v[k] = from < blocks ? partial[static_cast<int64_t>(from) * 2 * dim + at] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kSumAhead; ++k) sum += static_cast<double>(v[k]);
    }
    sums[row][column] = sum;
    __syncthreads();
    for (int half = kSumRows / 2; half >= 1; half /= 2) {
        if (row < half) {
            sum += sums[row + half][column];
            sums[row][column] = sum;
        }
        __syncthreads();
    }
    if (row != 0) return;
    W* const out = at < dim ? grad_q : grad_k;
    if (out) out[at < dim ? at : at - dim] = static_cast<W>(static_cast<float>(sum));
}

Steps steps_of(const actq_heads* q, const actq_heads* k, int lanes)
{
    const int side = 64 / lanes;
    Steps s;
    s.q_heads = q->heads;
    s.k_heads = k ? k->heads : 0;
    s.q = (s.q_heads + side - 1) / side;
    s.all = s.q + (s.k_heads + side - 1) / side;
    return s;
}

// Wavefronts that a pass is cut into where there are few tokens: 16 per compute unit [8192: alike; 2048: 1024 tokens 6.3 -> 6.9 us].
constexpr int64_t kNormUnits = 4096;
// Workgroups of the backward pass: two per compute unit, so that their shares of the weights' gradients stay few [256 and 1024 of them: 4095 tokens of
// 12 + 4 heads of 64 16.9 -> 19.4 and 21.6 us, 16384 of 32 + 8 of 128 92 -> 147 and 95].
constexpr int64_t kGradBlocks = 512;

int64_t grad_blocks(int64_t tokens)
{
    const int64_t need = (tokens + kNormWaves - 1) / kNormWaves;
    return need < kGradBlocks ? need : kGradBlocks;
}

}  // namespace

uint64_t head_norm_workspace(int64_t tokens, int32_t dim) { return static_cast<uint64_t>(grad_blocks(tokens)) * 2 * dim * sizeof(float); }

int launch_head_norm(const actq_heads* q, const actq_heads* k, int dtype, int64_t tokens, int32_t dim, const void* q_weight, const void* k_weight, int weight_dtype,
                     const actq_rotation* rotation, float eps, const actq_heads* q_out, const actq_heads* k_out, void* stream)
{
    return by_dtype(dtype, [&](auto type) {
        return by_dim(dim, [&](auto d) {
            typedef decltype(type) T;
            constexpr int kLanes = decltype(d)::value / kLaneValues;
            NormArgs<T> a = {};
            a.q = heads_of<T>(q);
            a.k = heads_of<T>(k);
            a.q_out = heads_of<T>(q_out);
            a.k_out = heads_of<T>(k_out);
            a.steps = steps_of(q, k, kLanes);
            a.tokens = tokens;
            const int64_t parts = kNormUnits / tokens < 1 ? 1 : kNormUnits / tokens < a.steps.all ? kNormUnits / tokens : a.steps.all;
            a.per_part = static_cast<uint32_t>((a.steps.all + parts - 1) / parts);
            a.parts = (a.steps.all + a.per_part - 1) / a.per_part;
            a.by_parts = make_fastdiv(a.parts);
            a.rotation = rotation_of(rotation);
            a.weights = {q_weight, k_weight, weight_dtype == ACTQ_F32};
            a.eps = eps;
            const uint64_t units = static_cast<uint64_t>(tokens) * a.parts;
            launch(head_norm_kernel<T, kLanes>, static_cast<unsigned>((units + kNormWaves - 1) / kNormWaves), kNormBlock, static_cast<hipStream_t>(stream), a);
            return launched("actq_head_norm_rotate");
        });
    });
}

int launch_head_norm_backward(const actq_heads* grad_q, const actq_heads* grad_k, const actq_heads* q, const actq_heads* k, int dtype, int64_t tokens, int32_t dim,
                              const void* q_weight, const void* k_weight, int weight_dtype, const actq_rotation* rotation, float eps, const actq_heads* q_out,
                              const actq_heads* k_out, void* grad_q_weight, void* grad_k_weight, void* workspace, void* stream)
{
    const char* who = "actq_head_norm_rotate_backward";
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool weights = grad_q_weight || grad_k_weight;
    const int64_t blocks = grad_blocks(tokens);
    if (blocks > 0) {
        const int rc = by_dtype(dtype, [&](auto type) {
            return by_dim(dim, [&](auto d) {
                typedef decltype(type) T;
                constexpr int kLanes = decltype(d)::value / kLaneValues;
                NormGradArgs<T> a = {};
                a.gq = heads_of<T>(grad_q);
                a.gk = heads_of<T>(grad_k);
                a.q = heads_of<T>(q);
                a.k = heads_of<T>(k);
                a.q_out = heads_of<T>(q_out);
                a.k_out = heads_of<T>(k_out);
                a.steps = steps_of(q, k, kLanes);
                a.tokens = tokens;
                a.rotation = rotation_of(rotation);
                a.weights = {q_weight, k_weight, weight_dtype == ACTQ_F32};
                a.eps = eps;
                a.partial = weights ? static_cast<float*>(workspace) : nullptr;
                launch(head_norm_backward_kernel<T, kLanes>, static_cast<unsigned>(blocks), kNormBlock, s, a);
                return launched(who);
            });
        });
        if (rc != ACTQ_OK) return rc;
    }
    if (!weights) return ACTQ_OK;
    return by_dtype(weight_dtype, [&](auto type) {
        typedef decltype(type) W;
        launch(head_norm_weights_kernel<W>, 2 * dim / kSumColumns, kSumColumns * kSumRows, s, static_cast<const float*>(workspace), static_cast<int32_t>(blocks), dim,
               static_cast<W*>(grad_q_weight), static_cast<W*>(grad_k_weight));
        return launched(who);
    });
}

}  // namespace actq
