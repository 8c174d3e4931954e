// The norms behind and before a block of a residual network with its gate, its scale and the residual sum, and their gradients.
//
//   n = h t p,  t = (mean(h^2) + eps)^(-1/2)      over the `width` elements of a token; without p: n = h
//   r = x + scale g n                             without h: r = x
//   y = r q w,  q = (mean(r^2) + eps)^(-1/2)
// and with u the gradient of y, e that of r:
//   grad_x = e + q (u w - r q^2 mean(u w r)),  grad_w = sum over tokens of u r q
//   s = scale grad_x;  grad_g = s n;  grad_h = t (s g p - h t^2 mean(s g p h)) or s g;  grad_p = sum over tokens of s g h t
//
// What bounds it: memory.  A pass reads and writes every row once: a row lies in the registers of its team (a wavefront, or the
// wavefronts of a workgroup) between the loads, the two sums over it, one behind the other, and the stores.  All arithmetic is binary32;
// y comes from the sum r before r is rounded, so that each result is rounded once.
//
// Measured on one MI355X, whose copy of 1 GiB reaches 5.1 TB/s: 8192 tokens of 4096 in binary16 43 us (6.2 TB/s, some of it from the caches), eight tokens 3.8 us; gradients
// of 16384 tokens in bfloat16 157 + 6 us (5.1 TB/s), of 1023 tokens of 2047 in binary32 20 + 7 us (2.5 TB/s: rows that start at any element; of 2048, from the host, 19.9 instead of 26.2 us
// for both kernels).  binary32: 8192 tokens of 4096 99 us (5.4 TB/s), gradients of as many 165 us (4.9 TB/s).
#include "actq_heads.h"

namespace actq {
namespace {

template <typename T>
struct Rows {
    T* p;
    int64_t stride;   // in elements
};

template <typename T>
Rows<T> rows_of(const actq_rows* r)
{
    if (!r) return {nullptr, 0};
    return {static_cast<T*>(r->data), r->stride};
}

// Eight neighbouring elements of a row; zeros beyond its end.
template <typename T>
__device__ __forceinline__ void load_part(Eight<T>& e, const T* row, int first, int width)
{
    if (first + kLaneValues <= width) {
        e.load(row + first);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = first + i < width ? row[first + i] : static_cast<T>(0.0f);
}

template <typename T>
__device__ __forceinline__ void store_part(const Eight<T>& e, T* row, int first, int width)
{
    if (first + kLaneValues <= width) {
        e.store(row + first);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (first + i < width) row[first + i] = e.v[i];
}

// Eight elements of a vector for the channels, of the rows' type or binary32.
template <typename T>
__device__ __forceinline__ void load_channels(const void* v, int wide, int first, int width, float (&f)[8])
{
    if (wide) {
        Eight<float> e;
        load_part(e, static_cast<const float*>(v), first, width);
        e.widen(f);
    } else {
        Eight<T> e;
        load_part(e, static_cast<const T*>(v), first, width);
        e.widen(f);
    }
}

// Sums over a team in all its lanes, of several values at a time.  The wavefronts' shares go through one of two places in turn: who writes a
// place again has passed the barrier behind which all have read it.
template <int WAVES, int COUNT>
struct Team {
    float shares[2][WAVES][COUNT];

    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N], int& turn)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = sum_over_lanes<64>(v[i]);
        if (WAVES == 1) return;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) shares[turn][threadIdx.x / 64][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[i] += shares[turn][w][i];
        }
        turn ^= 1;
    }
};

constexpr int kSmallTeams = 4;   // teams of one wavefront in a workgroup

template <int WAVES>
constexpr int kBlockThreads = 64 * (WAVES == 1 ? kSmallTeams : WAVES);

template <typename T>
struct BlockArgs {
    Rows<T> x, h, gates, r, y;
    const void* weight;
    const void* post_weight;
    const void* gate;
    int32_t wide;
    int64_t tokens, first;   // first: workgroups of earlier launches
    int32_t width;
    float mean;   // 1 / width
    float scale, eps;
};

template <typename T, int WAVES, int PARTS>
__global__ __launch_bounds__(kBlockThreads<WAVES>) void block_norm_kernel(BlockArgs<T> a)
{
    __shared__ Team<WAVES, 1> team;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = WAVES == 1 ? threadIdx.x % 64 : threadIdx.x;
    const int64_t block = a.first + blockIdx.x, token = WAVES == 1 ? block * kSmallTeams + wave : block;
    if (WAVES == 1 && token >= a.tokens) return;
    int turn = 0;
    float r[PARTS][8];
    {
        Eight<T> ex[PARTS], eh[PARTS], eg[PARTS];
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
            const int first = kLaneValues * (lane + c * 64 * WAVES);
            load_part(ex[c], a.x.p + token * a.x.stride, first, a.width);
            if (a.h.p) load_part(eh[c], a.h.p + token * a.h.stride, first, a.width);
            if (a.gates.p) load_part(eg[c], a.gates.p + token * a.gates.stride, first, a.width);
        }
#pragma unroll
        for (int c = 0; c < PARTS; ++c) ex[c].widen(r[c]);
        if (a.h.p) {
            float n[PARTS][8];
#pragma unroll
            for (int c = 0; c < PARTS; ++c) eh[c].widen(n[c]);
            if (a.post_weight) {
                float square[1] = {0.0f};
#pragma unroll
                for (int c = 0; c < PARTS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) square[0] = fmaf(n[c][i], n[c][i], square[0]);
                team.sum(square, turn);
                const float t = 1.0f / sqrtf(fmaf(square[0], a.mean, a.eps));
#pragma unroll
                for (int c = 0; c < PARTS; ++c) {
                    float p[8];
                    load_channels<T>(a.post_weight, a.wide, kLaneValues * (lane + c * 64 * WAVES), a.width, p);
#pragma unroll
                    for (int i = 0; i < 8; ++i) n[c][i] = n[c][i] * t * p[i];
                }
            }
            if (a.gates.p || a.gate) {
#pragma unroll
                for (int c = 0; c < PARTS; ++c) {
                    float g[8];
                    if (a.gates.p)
                        eg[c].widen(g);
                    else
                        load_channels<T>(a.gate, a.wide, kLaneValues * (lane + c * 64 * WAVES), a.width, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) n[c][i] *= g[i];
                }
            }
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r[c][i] = fmaf(a.scale, n[c][i], r[c][i]);
                ex[c].round(r[c]);
                store_part(ex[c], a.r.p + token * a.r.stride, kLaneValues * (lane + c * 64 * WAVES), a.width);
            }
        }
    }
    float square[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < PARTS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) square[0] = fmaf(r[c][i], r[c][i], square[0]);
    team.sum(square, turn);
    const float q = 1.0f / sqrtf(fmaf(square[0], a.mean, a.eps));
#pragma unroll
    for (int c = 0; c < PARTS; ++c) {
        const int first = kLaneValues * (lane + c * 64 * WAVES);
        float w[8];
        load_channels<T>(a.weight, a.wide, first, a.width, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = r[c][i] * q * w[i];
        Eight<T> e;
        e.round(w);
        store_part(e, a.y.p + token * a.y.stride, first, a.width);
    }
}

template <typename T>
struct BlockGradArgs {
    Rows<T> er, ey, r, h, gates;          // gradients of r (or null) and y, the inputs
    Rows<T> x_out, h_out, gates_out;      // gradients of x, h and the tokens' gates
    const void* weight;
    const void* post_weight;
    const void* gate;
    int32_t wide;
    int64_t tokens;
    int32_t width;
    float mean;
    float scale, eps;
    float* partial;   // [workgroups][weight, post_weight, gate][width], those that are wanted; null: none
    int32_t of_post, of_gate, vectors;   // their places (post_weight, gate: -1 without one), how many there are
};

// A team goes through the tokens with the grid's stride and keeps its share of the channels' gradients in registers, beside the channels themselves and the next
// token's rows, which are on their way while one is worked on (but for teams of 16 wavefronts, which have half the registers); the teams of a workgroup join theirs in the LDS in a fixed order, a second kernel those of the workgroups.
template <typename T, int WAVES, int PARTS>
__global__ __launch_bounds__(kBlockThreads<WAVES>, WAVES == 16 ? 4 : 2) void block_norm_backward_kernel(BlockGradArgs<T> a)
{
    constexpr int kTeams = WAVES == 1 ? kSmallTeams : 1;
    __shared__ Team<WAVES, 3> team;
    __shared__ float joined[WAVES == 1 ? kSmallTeams * 64 * PARTS * 8 : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = WAVES == 1 ? threadIdx.x % 64 : threadIdx.x;
    const bool gated = a.gates.p || a.gate;
    int turn = 0;
    float grad_w[PARTS][8], grad_p[PARTS][8], grad_g[PARTS][8], weight[PARTS][8], post[PARTS][8], gate[PARTS][8];
    constexpr bool kHeld = WAVES < 16;
    const auto channels = [&] {
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
            const int first = kLaneValues * (lane + c * 64 * WAVES);
            load_channels<T>(a.weight, a.wide, first, a.width, weight[c]);
            if (a.gate) load_channels<T>(a.gate, a.wide, first, a.width, gate[c]);
            if (a.post_weight) {
                load_channels<T>(a.post_weight, a.wide, first, a.width, post[c]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) post[c][i] = 1.0f;
            }
        }
    };
    if (kHeld) channels();
#pragma unroll
    for (int c = 0; c < PARTS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) grad_w[c][i] = grad_p[c][i] = grad_g[c][i] = 0.0f;
    struct Token {
        Eight<T> e[PARTS], u[PARTS], r[PARTS], h[PARTS], g[PARTS];
    };
    const auto load = [&](Token& t, int64_t token) {
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
            const int first = kLaneValues * (lane + c * 64 * WAVES);
            t.e[c].v = {};
            t.h[c].v = {};
            load_part(t.u[c], a.ey.p + token * a.ey.stride, first, a.width);
            load_part(t.r[c], a.r.p + token * a.r.stride, first, a.width);
            if (a.er.p) load_part(t.e[c], a.er.p + token * a.er.stride, first, a.width);
            if (a.h.p) load_part(t.h[c], a.h.p + token * a.h.stride, first, a.width);
            if (a.gates.p) load_part(t.g[c], a.gates.p + token * a.gates.stride, first, a.width);
        }
    };
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kTeams;
    int64_t token = static_cast<int64_t>(blockIdx.x) * kTeams + (WAVES == 1 ? wave : 0);
    Token now;
    if (kHeld && token < a.tokens) load(now, token);
    for (; token < a.tokens; token += stride) {
        Token next;
        if (kHeld) {
            if (token + stride < a.tokens) load(next, token + stride);
        } else {
            load(now, token);
            channels();
        }
        float s[PARTS][8];
        float sums[3] = {0.0f, 0.0f, 0.0f};   // of r^2, u w r, h^2
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
            float u[8], r[8], h[8];
            now.u[c].widen(u);
            now.r[c].widen(r);
            now.h[c].widen(h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sums[0] = fmaf(r[i], r[i], sums[0]);
                sums[1] = fmaf(u[i] * weight[c][i], r[i], sums[1]);
                sums[2] = fmaf(h[i], h[i], sums[2]);
            }
        }
        team.sum(sums, turn);
        const float q = 1.0f / sqrtf(fmaf(sums[0], a.mean, a.eps));
        const float back = sums[1] * a.mean * q * q;
        const float t = a.post_weight ? 1.0f / sqrtf(fmaf(sums[2], a.mean, a.eps)) : 1.0f;
        // the gradient of x, and s: times the scale
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
            float u[8], r[8], e[8];
            now.u[c].widen(u);
            now.r[c].widen(r);
            now.e[c].widen(e);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                grad_w[c][i] = fmaf(u[i], r[i] * q, grad_w[c][i]);
                e[i] = fmaf(q, fmaf(-r[i], back, u[i] * weight[c][i]), e[i]);
                s[c][i] = a.scale * e[i];
            }
            Eight<T> out;
            out.round(e);
            store_part(out, a.x_out.p + token * a.x_out.stride, kLaneValues * (lane + c * 64 * WAVES), a.width);
        }
        if (a.h.p) {
            float along[1] = {0.0f};   // of s g p h
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
                float h[8];
                now.h[c].widen(h);
                if (gated) {
                    float g[8], gradient[8];
                    if (a.gates.p) {
                        now.g[c].widen(g);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) g[i] = gate[c][i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        gradient[i] = s[c][i] * (h[i] * t * post[c][i]);
                        s[c][i] *= g[i];
                    }
                    if (a.gates.p) {
                        Eight<T> out;
                        out.round(gradient);
                        store_part(out, a.gates_out.p + token * a.gates_out.stride, kLaneValues * (lane + c * 64 * WAVES), a.width);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) grad_g[c][i] += gradient[i];
                    }
                }
                if (a.post_weight) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        grad_p[c][i] = fmaf(s[c][i], h[i] * t, grad_p[c][i]);
                        s[c][i] *= post[c][i];
                        along[0] = fmaf(s[c][i], h[i], along[0]);
                    }
                }
            }
            if (a.post_weight) {
                team.sum(along, turn);
                const float towards = along[0] * a.mean * t * t;
#pragma unroll
                for (int c = 0; c < PARTS; ++c) {
                    float h[8];
                    now.h[c].widen(h);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[c][i] = t * fmaf(-h[i], towards, s[c][i]);
                }
            }
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
                Eight<T> out;
                out.round(s[c]);
                store_part(out, a.h_out.p + token * a.h_out.stride, kLaneValues * (lane + c * 64 * WAVES), a.width);
            }
        }
        if (kHeld) now = next;
    }
    if (!a.partial) return;
    const auto keep = [&](const float (&grad)[PARTS][8], int place) {
        float* const to = a.partial + (static_cast<int64_t>(blockIdx.x) * a.vectors + place) * a.width;
        if (WAVES == 1) {
            __syncthreads();   // the vector before has been read
#pragma unroll
            for (int c = 0; c < PARTS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) joined[(wave * PARTS + c) * 512 + kLaneValues * lane + i] = grad[c][i];
            __syncthreads();
            for (int i = threadIdx.x; i < a.width; i += 64 * kSmallTeams) {
                const float* const at = joined + i;
                to[i] = (at[0] + at[512 * PARTS]) + (at[2 * 512 * PARTS] + at[3 * 512 * PARTS]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
                Eight<float> e;
                e.round(grad[c]);
                store_part(e, to, kLaneValues * (lane + c * 64 * WAVES), a.width);
            }
        }
    };
    keep(grad_w, 0);
    if (a.of_post >= 0) keep(grad_p, a.of_post);
    if (a.of_gate >= 0) keep(grad_g, a.of_gate);
}

// The channels' gradients: the workgroups' shares in binary64.  A thread takes four columns of a 16th or 64th of the shares, all of its loads in flight: 64 columns a
// workgroup where there are many, 16 else (12288 columns of 512 shares 6.4 us, with 16 columns in steps of 4 bytes 12.7; 4094 columns 12.4 and 7).
constexpr int kSumThreads = 256;

template <typename W, int kSumColumns>
__global__ __launch_bounds__(kSumThreads) void block_channels_kernel(const float* partial, int32_t blocks, int32_t width, int32_t columns, W* first, W* second, W* third)
{
    constexpr int kSumRows = kSumThreads * 4 / kSumColumns, kSumAhead = 512 / kSumRows < 16 ? 512 / kSumRows : 16;
    __shared__ double sums[kSumRows][kSumColumns];
    const int quad = threadIdx.x % (kSumColumns / 4) * 4, row = threadIdx.x / (kSumColumns / 4), at = blockIdx.x * kSumColumns + quad;
    double sum[4] = {};
    for (int b = row; b < blocks; b += kSumRows * kSumAhead) {
        f32x4 v[kSumAhead];
#pragma unroll
        for (int k = 0; k < kSumAhead; ++k) {
            typedef f32x4 any __attribute__((aligned(4)));
            const int from = b + k * kSumRows;
            const float* const p = partial + static_cast<int64_t>(from) * columns + at;
            v[k] = f32x4{};
            if (from < blocks && at + 4 <= columns) {
                v[k] = *reinterpret_cast<const any*>(p);
            } else if (from < blocks) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (at + i < columns) v[k][i] = p[i];
            }
        }
#pragma unroll
        for (int k = 0; k < kSumAhead; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += static_cast<double>(v[k][i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[row][quad + i] = sum[i];
    __syncthreads();
    if (threadIdx.x >= kSumColumns) return;
    const int column = blockIdx.x * kSumColumns + threadIdx.x;
    if (column >= columns) return;
    double all = 0.0;
#pragma unroll
    for (int r = 0; r < kSumRows; ++r) all += sums[r][threadIdx.x];
    const int vector = column / width;
    W* const out = vector == 0 ? first : vector == 1 ? second : third;
    out[column - vector * width] = static_cast<W>(static_cast<float>(all));
}

template <int N>
using Number = std::integral_constant<int, N>;

// f(wavefronts of a team, parts of eight elements a lane).  Where there are few rows the launch is bound by the trips to memory of one: more wavefronts then
// have fewer loads each.
template <typename F>
int by_width(int32_t width, bool few, F f)
{
    if (width <= 512) return f(Number<1>{}, Number<1>{});
    if (few) return width <= 2048 ? f(Number<4>{}, Number<1>{}) : width <= 4096 ? f(Number<8>{}, Number<1>{}) : width <= 8192 ? f(Number<16>{}, Number<1>{}) : f(Number<16>{}, Number<2>{});
    if (width <= 1024) return f(Number<1>{}, Number<2>{});
    if (width <= 2048) return f(Number<1>{}, Number<4>{});
    return width <= 4096 ? f(Number<4>{}, Number<2>{}) : width <= 8192 ? f(Number<4>{}, Number<4>{}) : f(Number<16>{}, Number<2>{});
}

// A team's registers hold 16 columns a lane of 16-bit types, 8 of binary32.
template <typename T, typename F>
int by_width_backward(int32_t width, F f)
{
    if (width <= 512) return f(Number<1>{}, Number<1>{});
    if (width <= 2048) return f(Number<4>{}, Number<1>{});
    if (width > 8192) return f(Number<16>{}, Number<2>{});
    if constexpr (sizeof(T) == 4) return width <= 4096 ? f(Number<8>{}, Number<1>{}) : f(Number<16>{}, Number<1>{});
    else return width <= 4096 ? f(Number<4>{}, Number<2>{}) : f(Number<8>{}, Number<2>{});
}

constexpr int64_t kFewRows = 512;

// Workgroups of the backward pass: two per compute unit, so that their shares of the channels' gradients stay few.
constexpr int64_t kGradBlocks = 512;

int64_t grad_blocks(const actq_block* b)
{
    const int64_t teams = b->width <= 512 ? kSmallTeams : 1, need = (b->tokens + teams - 1) / teams;
    return need < kGradBlocks ? need : kGradBlocks;
}

int vectors_of(const actq_block* b) { return 1 + (b->post_weight != nullptr) + (b->gate != nullptr); }

}  // namespace

uint64_t block_norm_workspace(const actq_block* b) { return static_cast<uint64_t>(grad_blocks(b)) * vectors_of(b) * b->width * sizeof(float); }

int launch_block_norm(const actq_block* b, const actq_rows* x, const actq_rows* h, const actq_rows* r, const actq_rows* y, void* stream)
{
    return by_dtype(b->dt, [&](auto type) {
        return by_width(b->width, b->tokens < kFewRows, [&](auto waves, auto parts) {
            typedef decltype(type) T;
            constexpr int kWaves = decltype(waves)::value, kParts = decltype(parts)::value;
            BlockArgs<T> a = {};
            a.x = rows_of<T>(x);
            a.h = rows_of<T>(h);
            a.gates = rows_of<T>(b->gates);
            a.r = rows_of<T>(r);
            a.y = rows_of<T>(y);
            a.weight = b->weight;
            a.post_weight = b->post_weight;
            a.gate = b->gate;
            a.wide = b->weight_dt == ACTQ_F32;
            a.tokens = b->tokens;
            a.width = b->width;
            a.mean = 1.0f / static_cast<float>(b->width);
            a.scale = b->scale;
            a.eps = b->eps;
            const int64_t blocks = kWaves == 1 ? (b->tokens + kSmallTeams - 1) / kSmallTeams : b->tokens;
            launches(blocks, kBlockThreads<kWaves>, [&](int64_t first, unsigned count) {
                a.first = first;
                launch(block_norm_kernel<T, kWaves, kParts>, count, kBlockThreads<kWaves>, static_cast<hipStream_t>(stream), a);
            });
            return launched("actq_block_norm");
        });
    });
}

int launch_block_norm_backward(const actq_block* b, const actq_rows* grad_r, const actq_rows* grad_y, const actq_rows* r, const actq_rows* h, const actq_rows* grad_x,
                               const actq_rows* grad_h, const actq_rows* grad_gates, void* grad_weight, void* grad_post_weight, void* grad_gate, void* workspace, void* stream)
{
    const char* who = "actq_block_norm_backward";
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t blocks = grad_blocks(b);
    const int vectors = vectors_of(b);
    if (blocks > 0) {
        const int rc = by_dtype(b->dt, [&](auto type) {
            typedef decltype(type) T;
            return by_width_backward<T>(b->width, [&](auto waves, auto parts) {
                constexpr int kWaves = decltype(waves)::value, kParts = decltype(parts)::value;
                BlockGradArgs<T> a = {};
                a.er = rows_of<T>(grad_r);
                a.ey = rows_of<T>(grad_y);
                a.r = rows_of<T>(r);
                a.h = rows_of<T>(h);
                a.gates = rows_of<T>(b->gates);
                a.x_out = rows_of<T>(grad_x);
                a.h_out = rows_of<T>(grad_h);
                a.gates_out = rows_of<T>(grad_gates);
                a.weight = b->weight;
                a.post_weight = b->post_weight;
                a.gate = b->gate;
                a.wide = b->weight_dt == ACTQ_F32;
                a.tokens = b->tokens;
                a.width = b->width;
                a.mean = 1.0f / static_cast<float>(b->width);
                a.scale = b->scale;
                a.eps = b->eps;
                a.partial = grad_weight ? static_cast<float*>(workspace) : nullptr;
                a.of_post = b->post_weight ? 1 : -1;
                a.of_gate = b->gate ? vectors - 1 : -1;
                a.vectors = vectors;
                launch(block_norm_backward_kernel<T, kWaves, kParts>, static_cast<unsigned>(blocks), kBlockThreads<kWaves>, s, a);
                return launched(who);
            });
        });
        if (rc != ACTQ_OK) return rc;
    }
    if (!grad_weight) return ACTQ_OK;
    return by_dtype(b->weight_dt, [&](auto type) {
        typedef decltype(type) W;
        W* const outs[3] = {static_cast<W*>(grad_weight), static_cast<W*>(b->post_weight ? grad_post_weight : grad_gate), static_cast<W*>(grad_gate)};
        const int32_t columns = vectors * b->width;
        const auto sum = [&](auto wide) {
            constexpr int kColumns = decltype(wide)::value;
            launch(block_channels_kernel<W, kColumns>, static_cast<unsigned>((columns + kColumns - 1) / kColumns), kSumThreads, s, static_cast<const float*>(workspace),
                   static_cast<int32_t>(blocks), b->width, columns, outs[0], outs[1], outs[2]);
        };
        if (columns >= 8192)
            sum(Number<64>{});
        else
            sum(Number<16>{});
        return launched(who);
    });
}

}  // namespace actq
