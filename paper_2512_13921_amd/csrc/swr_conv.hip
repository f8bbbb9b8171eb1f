// swr_conv.hip -- short causal depthwise convolution on gfx950, forward and backward.
//
//     pre[t] = bias + sum_k w[k] x[t - K + 1 + k];     y = pre sigma(pre)  (or pre)
//     g = dy sigma (1 + pre (1 - sigma));   dx[t] = sum_k w[k] g[t + K - 1 - k];
//     dw[k] = sum_t g[t] x[t - K + 1 + k];  dbias = sum_t g[t]
//
// A thread has 16 bytes of channels of a run of tokens: weights in registers, the
// last K - 1 rows of x (and of g) in a window that moves along, so that every row is
// loaded once but for the K - 1 before (and after) the run.
//
// What bounds it is the bytes.
#include <algorithm>

#include "swr_lm_launch.h"
#include "swr_vectors.h"

namespace swr {
namespace {

constexpr int kRun = 16;            // tokens of a thread, forward
constexpr int kBackRun = 32;        // ... backward
constexpr int kGroup = 8;           // rows loaded ahead
constexpr int kBackGroup = 4;
constexpr int64_t kMostY = 32768;   // blocks of a launch in y, which take units in turn

__device__ inline float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * v));
}

__device__ inline int64_t tokens_of(const ConvParams& p, int64_t b) {
    return p.lengths ? min(max((int64_t)p.lengths[b], (int64_t)0), p.T) : p.T;
}

// A channel's weights, and its bias.
template <class E, int K>
struct Taps {
    float w[E::NE][K], bias[E::NE];
    __device__ Taps(const ConvParams& p, int64_t c) {
        const typename E::store* row = (const typename E::store*)p.w + c * K;
#pragma unroll
        for (int i = 0; i < E::NE; ++i) {
            const bool there = c + i < p.C;
#pragma unroll
            for (int k = 0; k < K; ++k) w[i][k] = there ? E::one(row[i * K + k]) : 0.0f;
            bias[i] = there && p.bias ? E::one(((const typename E::store*)p.bias)[c + i]) : 0.0f;
        }
    }
};

// A block's threads: 1 << shift of them along the channels, the others along the units (runs of
// tokens, of batch after batch).
template <class E, int K>
__global__ __launch_bounds__(256) void swr_conv_kernel(ConvParams p, int shift, int64_t runs) {
    typedef typename E::store T;
    typedef Slice<E, E::NE> Row;
    const int64_t c = ((int64_t)blockIdx.x * (1 << shift) + (threadIdx.x & ((1 << shift) - 1))) * E::NE;
    if (c >= p.C) return;
    const int n = (int)min(p.C - c, (int64_t)E::NE);
    const Taps<E, K> taps(p, c);
    const int64_t per_block = 256 >> shift;
    for (int64_t u = blockIdx.y * per_block + (threadIdx.x >> shift); u < p.B * runs; u += gridDim.y * per_block) {
        const int64_t b = u / runs, first = (u - b * runs) * kRun, end = min(first + kRun, p.T), live = tokens_of(p, b);
        const T* x = (const T*)p.x + b * p.sx_b;
        T* y = (T*)p.y + b * p.sy_b + c;
        const T* state = p.state ? (const T*)p.state + b * (K - 1) * p.C : nullptr;
        // Rows t - K + 1 .. t of x; before the first token those of the state.
        Row window[K];
        const auto fetch = [&](int64_t t) {
            Row r = {};
            if (t >= 0) {
                if (t < live && t < end) r.load(x + t * p.sx_t, (int)c, (int)p.C);
            } else if (state && t >= 1 - K) {
                r.load(state + (K - 1 + t) * p.C, (int)c, (int)p.C);
            }
            return r;
        };
#pragma unroll
        for (int k = 0; k + 1 < K; ++k) window[k + 1] = fetch(first + k - K + 1);
        Row kept[K];   // the state's rows that the new state may still need
        if (K > 1 && p.state_out && first == 0) {
#pragma unroll
            for (int k = 0; k + 1 < K; ++k) {
                const int64_t t = live + k - K + 1;
                kept[k] = {};
                if (t >= 0) kept[k].load(x + t * p.sx_t, (int)c, (int)p.C);
                else if (state) kept[k].load(state + (K - 1 + t) * p.C, (int)c, (int)p.C);
            }
        }
        for (int64_t t = first; t < end; t += kGroup) {
            Row next[kGroup];
#pragma unroll
            for (int i = 0; i < kGroup; ++i) next[i] = fetch(t + i);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
#pragma unroll
                for (int k = 0; k + 1 < K; ++k) window[k] = window[k + 1];
                window[K - 1] = next[i];
                float f[E::NE];
#pragma unroll
                for (int e = 0; e < E::NE; ++e) {
                    float pre = taps.bias[e];
#pragma unroll
                    for (int k = 0; k < K; ++k) pre = fmaf(taps.w[e][k], window[k][e], pre);
                    f[e] = p.silu ? pre * sigmoid(pre) : pre;
                    if (t + i >= live) f[e] = 0.0f;
                }
                if (t + i < end) store<E, E::NE>(y + (t + i) * p.sy_t, n, f);
            }
        }
        if (K > 1 && p.state_out && first == 0) {
#pragma unroll
            for (int k = 0; k + 1 < K; ++k) {
                float f[E::NE];
#pragma unroll
                for (int e = 0; e < E::NE; ++e) f[e] = kept[k][e];
                store<E, E::NE>((T*)p.state_out + (b * (K - 1) + k) * p.C + c, n, f);
            }
        }
    }
}

// Backward.  A block's 64 threads along the channels take every gridDim.y-th four runs, one for each of
// its waves; the waves' shares of dw and dbias are added in LDS, in order, and written as one row of `partial`.
template <class E, int K>
__global__ __launch_bounds__(256) void swr_conv_back_kernel(ConvParams p, int64_t runs) {
    typedef typename E::store T;
    typedef Slice<E, E::NE> Row;
    __shared__ float share[64 * E::NE * (K + 1)];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * E::NE;
    const int n = (int)max(min(p.C - c, (int64_t)E::NE), (int64_t)0);
    float sums[E::NE][K + 1] = {};
    if (n > 0) {
        const Taps<E, K> taps(p, c);
        for (int64_t u = blockIdx.y * 4 + wave; u < p.B * runs; u += gridDim.y * 4) {
            const int64_t b = u / runs, first = (u - b * runs) * kBackRun, end = min(first + kBackRun, p.T);
            const int64_t live = tokens_of(p, b);
            const T* x = (const T*)p.x + b * p.sx_b;
            const T* dy = (const T*)p.dy + b * p.sy_b;
            T* dx = (T*)p.dx + b * p.sd_b + c;
            Row window[K];
            float g[K][E::NE] = {};   // of the tokens t - K + 1 .. t
            const auto fetch = [&](const T* rows, int64_t stride, int64_t t) {
                Row r = {};
                if (t >= 0 && t < live && t < end + K - 1) r.load(rows + t * stride, (int)c, (int)p.C);
                return r;
            };
#pragma unroll
            for (int k = 0; k + 1 < K; ++k) window[k + 1] = fetch(x, p.sx_t, first + k - K + 1);
            // The token t takes part in the gradients of x at t - K + 1 .. t.
            for (int64_t t = first; t < end + K - 1; t += kBackGroup) {
                Row xs[kBackGroup], ds[kBackGroup];
#pragma unroll
                for (int i = 0; i < kBackGroup; ++i) {
                    xs[i] = fetch(x, p.sx_t, t + i);
                    ds[i] = fetch(dy, p.sy_t, t + i);
                }
#pragma unroll
                for (int i = 0; i < kBackGroup; ++i) {
                    const bool there = t + i < live, own = t + i < end;
#pragma unroll
                    for (int k = 0; k + 1 < K; ++k) window[k] = window[k + 1];
                    window[K - 1] = xs[i];
                    float f[E::NE];
#pragma unroll
                    for (int e = 0; e < E::NE; ++e) {
                        float pre = taps.bias[e], v = ds[i][e];
#pragma unroll
                        for (int k = 0; k < K; ++k) pre = fmaf(taps.w[e][k], window[k][e], pre);
                        if (p.silu) {
                            const float gate = sigmoid(pre);
                            v *= gate * fmaf(pre, 1.0f - gate, 1.0f);
                        }
                        if (!there) v = 0.0f;
#pragma unroll
                        for (int k = 0; k + 1 < K; ++k) g[k][e] = g[k + 1][e];
                        g[K - 1][e] = v;
                        const float mine = own ? v : 0.0f;
#pragma unroll
                        for (int k = 0; k < K; ++k) sums[e][k] = fmaf(mine, window[k][e], sums[e][k]);
                        sums[e][K] += mine;
                        // dx[t - K + 1] = sum_k w[k] g[t - k]
                        f[e] = 0.0f;
#pragma unroll
                        for (int k = 0; k < K; ++k) f[e] = fmaf(taps.w[e][k], g[K - 1 - k][e], f[e]);
                    }
                    const int64_t at = t + i - K + 1;
                    if (at >= live) {
#pragma unroll
                        for (int e = 0; e < E::NE; ++e) f[e] = 0.0f;
                    }
                    if (at >= first && at < end) store<E, E::NE>(dx + at * p.sd_t, n, f);
                }
            }
        }
    }
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
        __syncthreads();
        if (wave == w) {
#pragma unroll
            for (int e = 0; e < E::NE; ++e)
#pragma unroll
                for (int k = 0; k <= K; ++k) {
                    float* s = share + (e * (K + 1) + k) * 64 + lane;
                    if (w > 0) sums[e][k] += *s;
                    *s = sums[e][k];
                }
        }
    }
    if (wave == 3) {
        float* out = p.partial + (blockIdx.y * p.C + c) * (K + 1);
#pragma unroll
        for (int e = 0; e < E::NE; ++e)
#pragma unroll
            for (int k = 0; k <= K; ++k)
                if (e < n) out[e * (K + 1) + k] = sums[e][k];
    }
}

// dw and dbias: the sums over the rows of partial.  64 columns a block, a quarter of the rows a wave.
__global__ __launch_bounds__(256) void swr_conv_sums_kernel(ConvParams p, int taps, int rows) {
    __shared__ float buf[4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t width = p.C * (taps + 1);
    for (int64_t first = (int64_t)blockIdx.x * 64; first < width; first += (int64_t)gridDim.x * 64) {
        const int64_t at = first + lane;
        float s = 0.0f;
        if (at < width) {
#pragma unroll 8
            for (int r = wave; r < rows; r += 4) s += p.partial[r * width + at];
        }
        buf[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && at < width) {
            s = (buf[0][lane] + buf[1][lane]) + (buf[2][lane] + buf[3][lane]);
            const int64_t c = at / (taps + 1);
            const int k = (int)(at - c * (taps + 1));
            if (k < taps) p.dw[c * taps + k] = s;
            else if (p.db) p.db[c] = s;
        }
        __syncthreads();
    }
}

template <template <class, int> class F, class E>
hipError_t by_taps(int taps, const F<E, 1>&, const ConvParams& p, hipStream_t st) {
    switch (taps) {
        case 1: return F<E, 1>::run(p, st);
        case 2: return F<E, 2>::run(p, st);
        case 3: return F<E, 3>::run(p, st);
        case 4: return F<E, 4>::run(p, st);
        case 5: return F<E, 5>::run(p, st);
        case 6: return F<E, 6>::run(p, st);
        case 7: return F<E, 7>::run(p, st);
        case 8: return F<E, 8>::run(p, st);
    }
    return hipErrorInvalidValue;
}

template <class E, int K>
struct Forward {
    static hipError_t run(const ConvParams& p, hipStream_t st) {
        const int64_t vectors = (p.C + E::NE - 1) / E::NE, runs = std::max<int64_t>(1, (p.T + kRun - 1) / kRun);
        int shift = 0;
        while (shift < 8 && ((int64_t)1 << shift) < vectors) ++shift;
        const int64_t units = (p.B * runs + (256 >> shift) - 1) / (256 >> shift);
        hipLaunchKernelGGL((swr_conv_kernel<E, K>),
                           dim3((unsigned)((vectors + (1 << shift) - 1) >> shift), (unsigned)std::min(units, kMostY)),
                           dim3(256), 0, st, p, shift, runs);
        return hipGetLastError();
    }
};

// Rows of partial sums: as many blocks as fill the GPU and no more than there are fours of runs.
int64_t back_rows(int64_t B, int64_t T, int64_t C, int ne) {
    const int64_t fours = (B * ((T + kBackRun - 1) / kBackRun) + 3) / 4, along = (C + 64 * ne - 1) / (64 * ne);
    return std::max<int64_t>(1, std::min(fours, std::max<int64_t>(1, (1536 + along - 1) / along)));
}

template <class E, int K>
struct Backward {
    static hipError_t run(const ConvParams& p, hipStream_t st) {
        const int64_t along = (p.C + 64 * E::NE - 1) / (64 * E::NE), rows = back_rows(p.B, p.T, p.C, E::NE);
        hipLaunchKernelGGL((swr_conv_back_kernel<E, K>), dim3((unsigned)along, (unsigned)rows), dim3(256), 0, st, p,
                           (p.T + kBackRun - 1) / kBackRun);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int64_t blocks = std::min<int64_t>((p.C * (K + 1) + 63) / 64, 1 << 20);
        hipLaunchKernelGGL(swr_conv_sums_kernel, dim3((unsigned)blocks), dim3(256), 0, st, p, K, (int)rows);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_conv(int dtype, int taps, const ConvParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    return dtype == SWR_DTYPE_F32 ? by_taps<Forward, F32>(taps, {}, p, st) : by_taps<Forward, Bf16>(taps, {}, p, st);
}

int64_t conv_work_bytes(int dtype, int64_t B, int64_t T, int64_t C, int taps) {
    return back_rows(B, T, C, dtype == SWR_DTYPE_F32 ? F32::NE : Bf16::NE) * C * (taps + 1) * 4;
}

hipError_t launch_conv_backward(int dtype, int taps, const ConvParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    return dtype == SWR_DTYPE_F32 ? by_taps<Backward, F32>(taps, {}, p, st) : by_taps<Backward, Bf16>(taps, {}, p, st);
}

}  // namespace swr
