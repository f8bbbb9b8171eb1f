// swr_conv.hip -- short causal depthwise convolution on gfx950, forward and backward.
//
//     pre[t] = bias + sum_k w[k] x[t - K + 1 + k];     y = pre sigma(pre)  (or pre)
//     g = dy sigma (1 + pre (1 - sigma));   dx[t] = sum_k w[k] g[t + K - 1 - k];
//     dw[k] = sum_t g[t] x[t - K + 1 + k];  dbias = sum_t g[t]
//
// A thread has four channels of a run of tokens: weights in registers, the
// last K - 1 rows of x (and of g) in a window that moves along, so that every row is
// loaded once but for the K - 1 before (and after) the run.
//
// What bounds it is the bytes: 5 x 4099 x 4096 bf16 with 4 taps take 72 us forward (336 MB, 4.7 TB/s) and 117
// backward (504 MB and the rows around the runs).  A single token is latency, 5.6 us for 64 x 4096.
#include <algorithm>
#include <type_traits>

#include "swr_lm_launch.h"
#include "swr_vectors.h"

namespace swr {
namespace {

constexpr int kRun = 16;            // tokens of a thread, forward
constexpr int kBackGroup = 4;       // tokens that the backward loads ahead
constexpr int64_t kMostY = 32768;   // blocks of a launch in y, which take units in turn

__device__ inline float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * v));
}

__device__ inline int64_t tokens_of(const ConvParams& p, int64_t b) {
    return p.lengths ? min(max((int64_t)p.lengths[b], (int64_t)0), p.T) : p.T;
}

// NE channels of a row as they lie in memory; without WHOLE as many of them as there are, and zeros.
template <class E, int NE>
struct Row {
    typedef typename E::store T;
    static constexpr int kWords = NE * (int)sizeof(T) / 4;
    struct __attribute__((packed, aligned(sizeof(T)))) Loose {
        uint32_t w[kWords];
    };
    uint32_t w[kWords];
    template <bool WHOLE>
    __device__ void load(const T* p, int n) {
        if constexpr (WHOLE) {
            const Loose v = *(const Loose*)p;
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = v.w[i];
        } else {
            T t[NE] = {};
#pragma unroll
            for (int i = 0; i < NE; ++i)
                if (i < n) t[i] = p[i];
            __builtin_memcpy(w, t, sizeof w);
        }
    }
    __device__ float operator[](int i) const {
        if constexpr (sizeof(T) == 4) return as_float(w[i]);
        else return as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    template <bool WHOLE>
    static __device__ void store(T* p, int n, const float* f) {
        T t[NE];
#pragma unroll
        for (int i = 0; i < NE; ++i) t[i] = E::to(f[i]);
        if constexpr (WHOLE) {
            Loose v;
            __builtin_memcpy(&v, t, sizeof v);
            *(Loose*)p = v;
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i)
                if (i < n) p[i] = t[i];
        }
    }
};

// A channel's weights, and its bias.
template <class E, int NE, int K>
struct Taps {
    float w[NE][K], bias[NE];
    __device__ Taps(const ConvParams& p, int64_t c) {
        const typename E::store* row = (const typename E::store*)p.w + c * K;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const bool there = c + i < p.C;
#pragma unroll
            for (int k = 0; k < K; ++k) w[i][k] = there ? E::one(row[i * K + k]) : 0.0f;
            bias[i] = there && p.bias ? E::one(((const typename E::store*)p.bias)[c + i]) : 0.0f;
        }
    }
};

// A block's threads: 1 << shift of them along the channels, the others along the units (runs of
// tokens, of batch after batch).  A whole run (of tokens and of channels) has no branches, so that its loads
// go ahead of its stores.
template <class E, int NE, int K, bool WHOLE, bool SILU>
__global__ __launch_bounds__(256) void swr_conv_kernel(ConvParams p, int shift, int64_t runs) {
    typedef typename E::store T;
    typedef Row<E, NE> R;
    const int64_t c = ((int64_t)blockIdx.x * (1 << shift) + (threadIdx.x & ((1 << shift) - 1))) * NE;
    if (c >= p.C) return;
    const int n = (int)min(p.C - c, (int64_t)NE);
    const Taps<E, NE, K> taps(p, c);
    const int64_t per_block = 256 >> shift;
    for (int64_t u = blockIdx.y * per_block + (threadIdx.x >> shift); u < p.B * runs; u += gridDim.y * per_block) {
        // (a division of 64 bits would cost a token alone as much as the rest)
        const int64_t b = p.B * runs >> 32 ? u / runs : (int64_t)((uint32_t)u / (uint32_t)runs);
        const int64_t first = (u - b * runs) * kRun, end = min(first + kRun, p.T), live = tokens_of(p, b);
        const T* x = (const T*)p.x + b * p.sx_b + c;
        T* y = (T*)p.y + b * p.sy_b + c;
        const T* state = p.state ? (const T*)p.state + b * (K - 1) * p.C + c : nullptr;
        // Rows before the run, of the state before the first token.
        R window[K];
#pragma unroll
        for (int k = 0; k + 1 < K; ++k) {
            const int64_t t = first + k - K + 1;
            window[k + 1] = {};
            if (t >= 0 && t < live) window[k + 1].template load<WHOLE>(x + t * p.sx_t, n);
            if (t < 0 && state) window[k + 1].template load<WHOLE>(state + (K - 1 + t) * p.C, n);
        }
        R kept[K];   // the state's rows that the new state may still need
        if (K > 1 && p.state_out && first == 0) {
#pragma unroll
            for (int k = 0; k + 1 < K; ++k) {
                const int64_t t = live + k - K + 1;
                kept[k] = {};
                if (t >= 0) kept[k].template load<WHOLE>(x + t * p.sx_t, n);
                else if (state) kept[k].template load<WHOLE>(state + (K - 1 + t) * p.C, n);
            }
        }
        const auto run = [&](auto whole) {
            constexpr bool kAll = whole;
            R rows[kRun];
#pragma unroll
            for (int i = 0; i < kRun; ++i)
                if (kAll || first + i < live) rows[i].template load<WHOLE>(x + (first + i) * p.sx_t, n);
                else rows[i] = {};
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
#pragma unroll
                for (int k = 0; k + 1 < K; ++k) window[k] = window[k + 1];
                window[K - 1] = rows[i];
                float f[NE];
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    float pre = taps.bias[e];
#pragma unroll
                    for (int k = 0; k < K; ++k) pre = fmaf(taps.w[e][k], window[k][e], pre);
                    f[e] = SILU ? pre * sigmoid(pre) : pre;
                    if (!kAll && first + i >= live) f[e] = 0.0f;
                }
                if (kAll || first + i < end) R::template store<WHOLE>(y + (first + i) * p.sy_t, n, f);
            }
        };
        if (first + kRun <= live) run(std::true_type());
        else run(std::false_type());
        if (K > 1 && p.state_out && first == 0) {
#pragma unroll
            for (int k = 0; k + 1 < K; ++k) {
                float f[NE];
#pragma unroll
                for (int e = 0; e < NE; ++e) f[e] = kept[k][e];
                R::template store<WHOLE>((T*)p.state_out + (b * (K - 1) + k) * p.C + c, n, f);
            }
        }
    }
}

// Backward.  A block's 64 threads along the channels, four channels each, take every gridDim.y-th four runs, one for
// each of its waves; the waves' shares of dw and dbias are added in LDS, in order, and written as one row of `partial`.
// (With eight bf16 channels a thread, of 272 registers, 5 x 4099 x 4096 took 274 us.)
template <class E, int NE, int K, bool WHOLE, bool SILU>
__global__ __launch_bounds__(256) void swr_conv_back_kernel(ConvParams p, int run, int64_t runs) {
    typedef typename E::store T;
    typedef Row<E, NE> R;
    __shared__ float share[64 * NE * (K + 1)];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * NE;
    // (Rows are a wave's: their addresses are scalars, a lane adds 32 bits.)
    const uint32_t bytes = (uint32_t)c * (uint32_t)sizeof(T);
    const auto at_lane = [&](auto* row) { return (decltype(row))((const char*)row + bytes); };
    const int n = (int)max(min(p.C - c, (int64_t)NE), (int64_t)0);
    float sums[NE][K + 1] = {};
    if (n > 0) {
        const Taps<E, NE, K> taps(p, c);
        for (int64_t u = blockIdx.y * 4 + wave; u < p.B * runs; u += gridDim.y * 4) {
            const int64_t b = u / runs;
            const int first = (int)(u - b * runs) * run, end = (int)min((int64_t)first + run, p.T);
            const int live = __builtin_amdgcn_readfirstlane((int)tokens_of(p, b));
            const T* x = (const T*)p.x + b * p.sx_b;
            const T* dy = (const T*)p.dy + b * p.sy_b;
            T* dx = (T*)p.dx + b * p.sd_b;
            if (first >= live) {   // nothing there
                const float zeros[NE] = {};
                for (int t = first; t < end; ++t) R::template store<WHOLE>(at_lane(dx + t * p.sd_t), n, zeros);
                continue;
            }
            R window[K];
            float g[K][NE] = {};   // of the tokens t - K + 1 .. t
#pragma unroll
            for (int k = 0; k + 1 < K; ++k) {
                const int t = first + k - K + 1;
                window[k + 1] = {};
                if (t >= 0) window[k + 1].template load<WHOLE>(at_lane(x + t * p.sx_t), n);
            }
            struct Group {
                R x[kBackGroup], dy[kBackGroup];
            } even, odd;
            // (Past the last token that counts that one once more: it comes from a cache.)
            const int last = min(live, end + K - 1) - 1;
            const auto fetch = [&](Group& v, int t) {
#pragma unroll
                for (int i = 0; i < kBackGroup; ++i) {
                    const int at = min(t + i, last);
                    v.x[i].template load<WHOLE>(at_lane(x + at * p.sx_t), n);
                    v.dy[i].template load<WHOLE>(at_lane(dy + at * p.sy_t), n);
                }
            };
            // The token t takes part in the gradients of x at t - K + 1 .. t.
            const auto step = [&](const Group& v, int t) {
#pragma unroll
                for (int i = 0; i < kBackGroup; ++i) {
                    const bool there = t + i <= last, own = t + i < end;
#pragma unroll
                    for (int k = 0; k + 1 < K; ++k) window[k] = window[k + 1];
                    window[K - 1] = v.x[i];
                    float f[NE];
#pragma unroll
                    for (int e = 0; e < NE; ++e) {
                        float pre = taps.bias[e], d = v.dy[i][e];
#pragma unroll
                        for (int k = 0; k < K; ++k) pre = fmaf(taps.w[e][k], window[k][e], pre);
                        if constexpr (SILU) {
                            const float gate = sigmoid(pre);
                            d *= gate * fmaf(pre, 1.0f - gate, 1.0f);
                        }
                        if (!there) d = 0.0f;
#pragma unroll
                        for (int k = 0; k + 1 < K; ++k) g[k][e] = g[k + 1][e];
                        g[K - 1][e] = d;
                        const float mine = own ? d : 0.0f;
#pragma unroll
                        for (int k = 0; k < K; ++k) {
                            // (past the run's tokens, or the last, the window's may be infinite, 0 times which is NaN)
                            const float xe = there && own ? window[k][e] : 0.0f;
                            sums[e][k] = fmaf(mine, xe, sums[e][k]);
                        }
                        sums[e][K] += mine;
                        // dx[t - K + 1] = sum_k w[k] g[t - k]
                        f[e] = 0.0f;
#pragma unroll
                        for (int k = 0; k < K; ++k) f[e] = fmaf(taps.w[e][k], g[K - 1 - k][e], f[e]);
                    }
                    const int at = t + i - K + 1;
                    if (at >= live) {
#pragma unroll
                        for (int e = 0; e < NE; ++e) f[e] = 0.0f;
                    }
                    if (at >= first && at < end) R::template store<WHOLE>(at_lane(dx + at * p.sd_t), n, f);
                }
            };
            fetch(even, first);
            for (int t = first; t < end + K - 1; t += 2 * kBackGroup) {
                fetch(odd, t + kBackGroup);
                step(even, t);
                fetch(even, t + 2 * kBackGroup);
                step(odd, t + kBackGroup);
            }
        }
    }
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
        __syncthreads();
        if (wave == w) {
#pragma unroll
            for (int e = 0; e < NE; ++e)
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
        for (int e = 0; e < NE; ++e)
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
        constexpr int NE = 4;
        const int64_t vectors = (p.C + NE - 1) / NE, runs = std::max<int64_t>(1, (p.T + kRun - 1) / kRun);
        int shift = 0;
        while (shift < 8 && ((int64_t)1 << shift) < vectors) ++shift;
        const int64_t units = (p.B * runs + (256 >> shift) - 1) / (256 >> shift);
        const dim3 grid((unsigned)((vectors + (1 << shift) - 1) >> shift), (unsigned)std::min(units, kMostY));
        const auto kernel = p.C % NE == 0 ? p.silu ? swr_conv_kernel<E, NE, K, true, true>
                                                   : swr_conv_kernel<E, NE, K, true, false>
                                          : p.silu ? swr_conv_kernel<E, NE, K, false, true>
                                                   : swr_conv_kernel<E, NE, K, false, false>;
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, p, shift, runs);
        return hipGetLastError();
    }
};

constexpr int kBackChannels = 4;   // of a thread

// Tokens of a run, backward: long ones load fewer rows twice, short ones are more.  By the waves that runs of 32 make:
// 1 x 2048 x 2048 (512 waves) takes 17.5 us in runs of 16, 23.1 of 32, 27.7 of 48; 8 x 1000 x 1000 (1024) 26.1, 23.7, 28.3;
// 2 x 2048 x 4096 (2048) 37.0, 32.0, 38.4; 5 x 4099 x 4096 (10320) 126 of 32, 117 of 48, 129 of 64.
int back_run(int64_t B, int64_t T, int64_t C) {
    const int64_t waves = B * ((T + 31) / 32) * ((C + 64 * kBackChannels - 1) / (64 * kBackChannels));
    return waves < 1024 ? 16 : waves < 8192 ? 32 : 48;
}
// Rows of partial sums: as many blocks as fill the GPU and no more than there are fours of runs.
int64_t back_rows(int64_t B, int64_t T, int64_t C) {
    const int run = back_run(B, T, C);
    const int64_t fours = (B * ((T + run - 1) / run) + 3) / 4, along = (C + 64 * kBackChannels - 1) / (64 * kBackChannels);
    return std::max<int64_t>(1, std::min(fours, std::max<int64_t>(1, (1024 + along - 1) / along)));
}

template <class E, int K>
struct Backward {
    static hipError_t run(const ConvParams& p, hipStream_t st) {
        constexpr int NE = kBackChannels;
        const int64_t along = (p.C + 64 * NE - 1) / (64 * NE), rows = back_rows(p.B, p.T, p.C);
        const int run = back_run(p.B, p.T, p.C);
        const int64_t runs = (p.T + run - 1) / run;
        const dim3 grid((unsigned)along, (unsigned)rows);
        const auto kernel = p.C % NE == 0 ? p.silu ? swr_conv_back_kernel<E, NE, K, true, true>
                                                   : swr_conv_back_kernel<E, NE, K, true, false>
                                          : p.silu ? swr_conv_back_kernel<E, NE, K, false, true>
                                                   : swr_conv_back_kernel<E, NE, K, false, false>;
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, p, run, runs);
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

int64_t conv_work_bytes(int64_t B, int64_t T, int64_t C, int taps) {
    return back_rows(B, T, C) * C * (taps + 1) * 4;
}

hipError_t launch_conv_backward(int dtype, int taps, const ConvParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    return dtype == SWR_DTYPE_F32 ? by_taps<Backward, F32>(taps, {}, p, st) : by_taps<Backward, Bf16>(taps, {}, p, st);
}

}  // namespace swr
