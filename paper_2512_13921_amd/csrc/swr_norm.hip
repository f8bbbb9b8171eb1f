// swr_norm.hip -- residual addition and root-mean-square norm, forward and
// backward, on gfx950.
//
//     h = x + r;   y = h rho w,   rho = 1 / sqrt(mean(h^2) + eps)
//     n = h rho, g = dy w:   dx = rho (g - n mean(g n)) + dh,   dw = sum_rows dy n
//
// Every tensor is moved once: a row is held in registers between the sum over it
// and its outputs, by a wave or a block of its own.  The forward's two row sums (h^2
// and, for 8-bit outputs, max|h w|) need the loads alone, so both are reduced
// together; so do the backward's (h^2 and g h).
//
// What bounds it is the bytes: 20495 rows of 2048 bf16 take 54 us forward and 77
// backward, 5.1 TB/s, where a copy reaches 5.2.  A few rows are bound by latency: 8 of
// 2048, with 8-bit output, 3.3 us.
#include <algorithm>

#include "swr_hybrid_launch.h"
#include "swr_vectors.h"

namespace swr {
namespace {

// Sums of a and b (or a's sum and b's maximum) over the threads of a row, a
// wave or (BLOCK) a whole block; every thread gets them, added in the same order.
// `buf` holds 2 values a wave.
template <bool BLOCK>
__device__ inline void row_sums(float& a, float& b, float* buf) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (BLOCK) {
        const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
        __syncthreads();   // (the last row's values have been read)
        if (threadIdx.x % 64 == 0) { buf[2 * wave] = a; buf[2 * wave + 1] = b; }
        __syncthreads();
        a = b = 0.0f;
        for (int i = 0; i < waves; ++i) { a += buf[2 * i]; b += buf[2 * i + 1]; }
    }
}
template <bool BLOCK>
__device__ inline void row_sum_max(float& a, uint32_t& b, float* buf) {
    a = wave_sum(a);
    b = wave_max(b);
    if constexpr (BLOCK) {
        const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
        __syncthreads();
        if (threadIdx.x % 64 == 0) { buf[2 * wave] = a; buf[2 * wave + 1] = __builtin_bit_cast(float, b); }
        __syncthreads();
        a = 0.0f;
        b = 0;
        for (int i = 0; i < waves; ++i) { a += buf[2 * i]; b = max(b, __builtin_bit_cast(uint32_t, buf[2 * i + 1])); }
    }
}

__device__ inline int64_t row_offset(int64_t row, uint32_t inner, int64_t so, int64_t si) {
    const uint32_t o = (uint32_t)row / inner;
    return o * so + ((uint32_t)row - o * inner) * si;
}

// The scale of an 8-bit row whose largest |y| has these bits, and how its
// values become codes: v = (y * pre) * inv.  (Of floats' absolute values the
// integers keep the order, and a NaN is the largest.)  pre keeps inv finite
// for rows near the smallest floats.
struct Codes {
    float scale, pre, inv;
    __device__ explicit Codes(float top) {
        scale = top * (1.0f / 448.0f);
        pre = top < 0x1p-100f ? 0x1p64f : 1.0f;
        inv = top > 0.0f ? 448.0f / (top * pre) : 0.0f;
        if (top != top) inv = top;
    }
    __device__ float operator()(float y) const {
        const float v = (y * pre) * inv;
        return v > 448.0f ? 448.0f : v < -448.0f ? -448.0f : v;   // (keeps NaN)
    }
};

template <int NE>
__device__ inline void store_codes(uint8_t* p, int n, const float* f) {
    uint32_t w[NE / 4];
#pragma unroll
    for (int i = 0; i < NE / 4; ++i) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], c, true);
    }
    if (n >= NE) {
        __builtin_memcpy(p, w, NE);
    } else if (n > 0) {
#pragma unroll
        for (int i = 0; i < NE - 1; ++i)
            if (i < n) p[i] = (uint8_t)(w[i / 4] >> 8 * (i % 4));
    }
}

// Most floats of a row that a thread holds, and most threads of a row's own
// block: with 1024 a thread has 128 registers, which hold 16 of the
// backward's columns (h, dy, dh, weight and dw) and four vectors of the forward's.
constexpr int kFloats = 32, kForwardThreads = 1024, kForwardVectors = 4;
constexpr int backward_threads(int floats) { return floats <= 16 ? 1024 : 512; }

// A row's threads: a wave of a block of four (rows of up to 64 VPT vectors of
// 16 bytes), or a block of as many waves as the row needs.
template <bool BLOCK>
struct Team {
    int t, size;       // this thread and the threads of a row
    int64_t row, step; // the team's first row, and from row to row
    __device__ Team()
        : t(BLOCK ? threadIdx.x : threadIdx.x % 64), size(BLOCK ? blockDim.x : 64),
          row(BLOCK ? blockIdx.x : (int64_t)blockIdx.x * 4 + threadIdx.x / 64),
          step(BLOCK ? gridDim.x : (int64_t)gridDim.x * 4) {}
    // First element of this thread's v-th vector of NE.
    template <int NE>
    __device__ int at(int v) const { return (v * size + t) * NE; }
};

template <class E, class WE, bool BLOCK, int VPT, bool FP8>
__global__ __launch_bounds__(BLOCK ? kForwardThreads : 256) void swr_norm_kernel(NormParams p) {
    constexpr int NE = E::NE;
    typedef typename E::store T;
    typedef typename WE::store WT;
    __shared__ float buf[32];
    const Team<BLOCK> team;
    for (int64_t row = team.row; row < p.rows; row += team.step) {
        const T* x = (const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i);
        const T* r = p.r ? (const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i) : nullptr;
        Slice<E, NE> xs[VPT], rs[VPT];
        Slice<WE, NE> ws[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) xs[v].load(x, team.template at<NE>(v), p.width);
        if (r) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) rs[v].load(r, team.template at<NE>(v), p.width);
        }
#pragma unroll
        for (int v = 0; v < VPT; ++v) ws[v].load((const WT*)p.w, team.template at<NE>(v), p.width);
        float h[VPT][NE], w[VPT][NE];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                h[v][i] = xs[v][i];
                w[v][i] = ws[v][i];
            }
            if (r) {
#pragma unroll
                for (int i = 0; i < NE; ++i) h[v][i] += rs[v][i];
            }
        }
        if (p.h) {
            T* ho = (T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i);
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                store<E, NE>(ho + team.template at<NE>(v), p.width - team.template at<NE>(v), h[v]);
        }
        float sum = 0.0f;
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                sum += h[v][i] * h[v][i];
                if constexpr (FP8) top = max(top, __builtin_bit_cast(uint32_t, h[v][i] * w[v][i]) & 0x7fffffffu);
            }
        if constexpr (FP8) {
            row_sum_max<BLOCK>(sum, top, buf);
        } else {
            float none = 0.0f;
            row_sums<BLOCK>(sum, none, buf);
        }
        const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
        const int64_t yo = row_offset(row, p.inner, p.sy_o, p.sy_i);
        if constexpr (FP8) {
            const Codes code(__builtin_bit_cast(float, top) * rho);
            if (team.t == 0) p.scale[row] = code.scale;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float f[NE];
#pragma unroll
                for (int i = 0; i < NE; ++i) f[i] = code(h[v][i] * w[v][i] * rho);
                store_codes<NE>((uint8_t*)p.y + yo + team.template at<NE>(v), p.width - team.template at<NE>(v), f);
            }
        } else {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float f[NE];
#pragma unroll
                for (int i = 0; i < NE; ++i) f[i] = h[v][i] * rho * w[v][i];
                store<E, NE>((T*)p.y + yo + team.template at<NE>(v), p.width - team.template at<NE>(v), f);
            }
        }
    }
}

// Rows too wide for registers (or narrower than a vector): 1024 threads walk a row
// twice, the second time out of the L2 or the 256 MB cache.  h is stored on the second walk, by the
// thread that reads the same element, so it may be x or the residual itself.
template <class E, class WE, bool FP8>
__global__ __launch_bounds__(1024) void swr_norm_wide_kernel(NormParams p) {
    constexpr int NE = E::NE;
    typedef typename E::store T;
    typedef typename WE::store WT;
    __shared__ float buf[32];
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = (const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i);
        const T* r = p.r ? (const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i) : nullptr;
        float sum = 0.0f;
        uint32_t top = 0;
        for (int64_t e = (int64_t)threadIdx.x * NE; e < p.width; e += 1024 * NE) {
            float h[NE], f[NE];
            load<E, NE>(x, (int)e, p.width, h);
            if (r) {
                load<E, NE>(r, (int)e, p.width, f);
#pragma unroll
                for (int i = 0; i < NE; ++i) h[i] += f[i];
            }
            if constexpr (FP8) load<WE, NE>((const WT*)p.w, (int)e, p.width, f);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                sum += h[i] * h[i];
                if constexpr (FP8) top = max(top, __builtin_bit_cast(uint32_t, h[i] * f[i]) & 0x7fffffffu);
            }
        }
        row_sum_max<true>(sum, top, buf);
        const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
        const Codes code(__builtin_bit_cast(float, top) * rho);
        if constexpr (FP8)
            if (threadIdx.x == 0) p.scale[row] = code.scale;
        T* ho = p.h ? (T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i) : nullptr;
        const int64_t yo = row_offset(row, p.inner, p.sy_o, p.sy_i);
        for (int64_t e = (int64_t)threadIdx.x * NE; e < p.width; e += 1024 * NE) {
            const int n = p.width - (int)e;
            float h[NE], f[NE];
            load<E, NE>(x, (int)e, p.width, h);
            if (r) {
                load<E, NE>(r, (int)e, p.width, f);
#pragma unroll
                for (int i = 0; i < NE; ++i) h[i] += f[i];
            }
            if (ho) store<E, NE>(ho + e, n, h);
            load<WE, NE>((const WT*)p.w, (int)e, p.width, f);
#pragma unroll
            for (int i = 0; i < NE; ++i) f[i] = FP8 ? code(h[i] * f[i] * rho) : h[i] * rho * f[i];
            if constexpr (FP8) store_codes<NE>((uint8_t*)p.y + yo + e, n, f);
            else store<E, NE>((T*)p.y + yo + e, n, f);
        }
    }
}

// Backward.  A row's threads take rows in turn and keep their columns'
// shares of dw in registers; a block joins its rows' shares in LDS, in order,
// and writes one row of `partial`, which swr_norm_dw_kernel sums.  A row's h, dy
// and dh are loaded together (with dh loaded after the sums, by a wave a row, 20495
// rows of 2048 bf16 took 116 us; 65 as it is, 5.1 TB/s).
template <class E, class WE, bool BLOCK, int VPT>
__global__ __launch_bounds__(BLOCK ? backward_threads(VPT * E::NE) : 256) void swr_norm_bwd_kernel(NormParams p) {
    constexpr int NE = E::NE;
    typedef typename E::store T;
    typedef typename WE::store WT;
    __shared__ float buf[32];
    __shared__ float share[BLOCK ? 1 : 64 * VPT * NE];
    const Team<BLOCK> team;
    struct {
        Slice<E, NE> h[VPT], dy[VPT], dh[VPT];
    } now, next;
    Slice<WE, NE> w[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) w[i].load((const WT*)p.w, team.template at<NE>(i), p.width);
    const auto fetch = [&](int64_t row, auto& v) {
        if (row >= p.rows) return;
        const T* h = (const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i);
        const T* dy = (const T*)p.y + row_offset(row, p.inner, p.sy_o, p.sy_i);
        const T* dh = p.r ? (const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i) : nullptr;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            v.h[i].load(h, team.template at<NE>(i), p.width);
            v.dy[i].load(dy, team.template at<NE>(i), p.width);
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (dh) v.dh[i].load(dh, team.template at<NE>(i), p.width);
            else v.dh[i] = {};
        }
    };
    float dw[VPT][NE] = {};
    if constexpr (!BLOCK) fetch(team.row, now);   // (a block's many waves hide its loads without)
    for (int64_t row = team.row; row < p.rows; row += team.step) {
        if constexpr (BLOCK) fetch(row, now);
        else fetch(row + team.step, next);
        float sum = 0.0f, along = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const float h = now.h[v][i];
                sum += h * h;
                along += now.dy[v][i] * w[v][i] * h;
            }
        }
        row_sums<BLOCK>(sum, along, buf);
        const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
        const float c = along / (float)p.width * rho * rho;   // mean(g n) rho, times h: n mean(g n)
        T* dx = (T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = team.template at<NE>(v), n = p.width - e;
            float f[NE];
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const float h = now.h[v][i], dy = now.dy[v][i];
                f[i] = now.dh[v][i] + rho * (dy * w[v][i] - h * c);
                dw[v][i] += dy * (h * rho);
            }
            store<E, NE>(dx + e, n, f);
        }
        if constexpr (!BLOCK) now = next;
    }
    float* out = p.partial + (int64_t)blockIdx.x * p.width;
    if constexpr (!BLOCK) {
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
            __syncthreads();
            if ((int)threadIdx.x / 64 == k) {
#pragma unroll
                for (int v = 0; v < VPT; ++v)
#pragma unroll
                    for (int i = 0; i < NE; ++i) {
                        float* s = share + (v * NE + i) * 64 + team.t;
                        if (k > 0) dw[v][i] += *s;
                        *s = dw[v][i];
                    }
            }
        }
    }
    if (BLOCK || threadIdx.x / 64 == 3) {
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            store<F32, NE>(out + team.template at<NE>(v), p.width - team.template at<NE>(v), dw[v]);
    }
}

// Wide rows' backward, first walk: 1 / rms and mean(g n) / rms of every row.
template <class E, class WE>
__global__ __launch_bounds__(1024) void swr_norm_stats_kernel(NormParams p) {
    constexpr int NE = E::NE;
    typedef typename E::store T;
    typedef typename WE::store WT;
    __shared__ float buf[32];
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* hr = (const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i);
        const T* dy = (const T*)p.y + row_offset(row, p.inner, p.sy_o, p.sy_i);
        float sum = 0.0f, along = 0.0f;
        for (int64_t e = (int64_t)threadIdx.x * NE; e < p.width; e += 1024 * NE) {
            float h[NE], d[NE], w[NE];
            load<E, NE>(hr, (int)e, p.width, h);
            load<E, NE>(dy, (int)e, p.width, d);
            load<WE, NE>((const WT*)p.w, (int)e, p.width, w);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                sum += h[i] * h[i];
                along += d[i] * w[i] * h[i];
            }
        }
        row_sums<true>(sum, along, buf);
        if (threadIdx.x == 0) {
            const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
            p.stats[row] = make_float2(rho, along / (float)p.width * rho * rho);
        }
    }
}

// Second walk: a block takes 256 vectors of columns (blockIdx.y and every gridDim.y-th) of
// every gridDim.x-th row.
template <class E, class WE>
__global__ __launch_bounds__(256) void swr_norm_bwd_wide_kernel(NormParams p) {
    constexpr int NE = E::NE;
    typedef typename E::store T;
    typedef typename WE::store WT;
    for (int64_t e = ((int64_t)blockIdx.y * 256 + threadIdx.x) * NE; e < p.width; e += (int64_t)gridDim.y * 256 * NE) {
        const int n = p.width - (int)e;
        float w[NE], dw[NE] = {};
        load<WE, NE>((const WT*)p.w, (int)e, p.width, w);
        for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
            const float2 s = p.stats[row];
            float h[NE], d[NE], f[NE] = {};
            load<E, NE>((const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i), (int)e, p.width, h);
            load<E, NE>((const T*)p.y + row_offset(row, p.inner, p.sy_o, p.sy_i), (int)e, p.width, d);
            if (p.r) load<E, NE>((const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i), (int)e, p.width, f);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                f[i] += s.x * (d[i] * w[i] - h[i] * s.y);
                dw[i] += d[i] * (h[i] * s.x);
            }
            store<E, NE>((T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i) + e, n, f);
        }
        store<F32, NE>(p.partial + (int64_t)blockIdx.x * p.width + e, n, dw);
    }
}

// dw: the sum of `blocks` rows of partial.  A block takes 16 columns (and 16 of every gridDim.x
// times 16 more), its 64 groups of 16 threads every 64th row, then the groups are added in order.
__global__ __launch_bounds__(1024) void swr_norm_dw_kernel(const float* partial, float* dw, int width, int blocks) {
    __shared__ float buf[64][16];
    const int c = threadIdx.x % 16, group = threadIdx.x / 16;
    for (int64_t first = (int64_t)blockIdx.x * 16; first < width; first += (int64_t)gridDim.x * 16) {
        const int64_t col = first + c;
        float s = 0.0f;
        if (col < width) {
#pragma unroll 8
            for (int b = group; b < blocks; b += 64) s += partial[(int64_t)b * width + col];
        }
        buf[group][c] = s;
        __syncthreads();
        if (group < 8) {
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += buf[8 * group + i][c];
            buf[8 * group][c] = s;
        }
        __syncthreads();
        if (group == 0 && col < width) {
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += buf[8 * i][c];
            dw[col] = s;
        }
        __syncthreads();   // (the sums have been read)
    }
}

constexpr int64_t kFewRows = 512;          // rows that leave a compute unit two or fewer: latency counts
constexpr int64_t kMostBlocks = 1 << 20;   // of a launch in x, whose blocks take rows (or columns) in turn
constexpr unsigned kMostColumns = 1 << 15; // of a launch in y, whose blocks take columns in turn

unsigned grid_of(int64_t blocks) { return (unsigned)std::min(blocks, kMostBlocks); }

template <int MOST, class F>
hipError_t by_vectors(int vpt, F f) {
    switch (vpt) {
        case 1: return f.template operator()<1>();
        case 2: if constexpr (MOST >= 2) return f.template operator()<2>(); break;
        case 4: if constexpr (MOST >= 4) return f.template operator()<4>(); break;
        case 8: if constexpr (MOST >= 8) return f.template operator()<8>(); break;
    }
    return hipErrorInvalidValue;
}

template <class E, class WE, bool BLOCK, bool FP8>
struct Forward {
    const NormPlan& plan;
    const NormParams& p;
    hipStream_t st;
    template <int VPT>
    hipError_t operator()() const {
        const int64_t teams = BLOCK ? p.rows : (p.rows + 3) / 4;
        hipLaunchKernelGGL((swr_norm_kernel<E, WE, BLOCK, VPT, FP8>), dim3(grid_of(teams)), dim3(plan.threads), 0, st,
                           p);
        return hipGetLastError();
    }
};

template <class E, class WE, bool BLOCK>
struct Backward {
    const NormPlan& plan;
    const NormParams& p;
    hipStream_t st;
    template <int VPT>
    hipError_t operator()() const {
        hipLaunchKernelGGL((swr_norm_bwd_kernel<E, WE, BLOCK, VPT>), dim3((unsigned)plan.blocks), dim3(plan.threads), 0,
                           st, p);
        return hipGetLastError();
    }
};

template <class E, class WE, bool FP8>
hipError_t held_forward(const NormPlan& plan, const NormParams& p, hipStream_t st) {
    return plan.block ? by_vectors<kForwardVectors>(plan.vpt, Forward<E, WE, true, FP8>{plan, p, st})
                      : by_vectors<1>(plan.vpt, Forward<E, WE, false, FP8>{plan, p, st});
}

template <class E, class WE>
hipError_t forward(const swr_norm_t& n, const NormPlan& plan, const NormParams& p, hipStream_t st) {
    const bool fp8 = n.out_dtype == SWR_DTYPE_FP8;
    if (plan.vpt > 0) return fp8 ? held_forward<E, WE, true>(plan, p, st) : held_forward<E, WE, false>(plan, p, st);
    if (fp8) hipLaunchKernelGGL((swr_norm_wide_kernel<E, WE, true>), dim3(grid_of(p.rows)), dim3(1024), 0, st, p);
    else hipLaunchKernelGGL((swr_norm_wide_kernel<E, WE, false>), dim3(grid_of(p.rows)), dim3(1024), 0, st, p);
    return hipGetLastError();
}

template <class E, class WE>
hipError_t backward(const NormPlan& plan, const NormParams& p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (p.rows == 0) {
        // (dw is a sum of nothing)
    } else if (plan.vpt == 0) {
        hipLaunchKernelGGL((swr_norm_stats_kernel<E, WE>), dim3(grid_of(p.rows)), dim3(1024), 0, st, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const unsigned cols = std::min((unsigned)((p.width + 256 * E::NE - 1) / (256 * E::NE)), kMostColumns);
        hipLaunchKernelGGL((swr_norm_bwd_wide_kernel<E, WE>), dim3((unsigned)plan.blocks, cols), dim3(256), 0, st, p);
        e = hipGetLastError();
    } else {
        e = plan.block ? by_vectors<kFloats / E::NE>(plan.vpt, Backward<E, WE, true>{plan, p, st})
                       : by_vectors<2>(plan.vpt, Backward<E, WE, false>{plan, p, st});
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(swr_norm_dw_kernel, dim3(grid_of((p.width + 15) / 16)), dim3(1024), 0, st, p.partial, p.dw,
                       p.width, plan.blocks);
    return hipGetLastError();
}

}  // namespace

// Waves of the backward that a SIMD holds, by the floats of a row that a thread
// has (its registers: 56 to 86, 112 to 128, 159 and more).
int waves_held(int floats) { return floats <= 8 ? 6 : floats <= 16 ? 4 : 2; }

// Rows of up to 64 vectors (128 in the backward, so that four rows share their
// sum of dw) are a wave's, wider ones a block's.  A thread takes as few vectors as
// keep a block within 512 threads (2 vectors: 768; the backward 768), since
// more, smaller waves hide the trips to memory: bf16 rows of 2048, forward, a
// block of 4 waves 47.6 us and a wave of 4 vectors 51.1 for 16384 of them; of 8192, 1, 2 and 4
// vectors 52.6, 51.9 and 50.6 forward, with 8-bit output 69.1, 49.7 and 52.2; of 16384, 2 and 4
// vectors 54.6 and 50.7.  The backward's blocks are those that a compute unit
// holds at once, and no more than about 16 waves of them, as each
// leaves a share of dw to be read again (rows of 2048, 28 waves 67.9 us and 7.9 for
// the shares, 16 waves 65.9 and 4.9).
NormPlan plan_norm(int dtype, int64_t rows, int64_t width, bool backward) {
    const int ne = dtype == SWR_DTYPE_BF16 ? Bf16::NE : F32::NE;
    const int64_t vectors = (width + ne - 1) / ne;
    NormPlan plan{false, 0, 0, 0};
    if (width < ne) {
        // (less than a vector: walked as the widest are)
    } else if (vectors <= 64 || (backward && rows > kFewRows && vectors <= 128)) {
        plan.vpt = vectors <= 64 ? 1 : 2;
        plan.threads = 256;
    } else {
        const int most = backward ? kFloats / ne : kForwardVectors;
        for (int vpt = 1; vpt <= most; vpt *= 2) {
            const int64_t threads = ((vectors + vpt - 1) / vpt + 63) / 64 * 64;
            if (threads > (backward ? backward_threads(vpt * ne) : kForwardThreads)) continue;
            // Is a block of fewer threads, with more vectors each, to be had and better?
            const bool more = backward ? 2 * vpt * ne <= 16 : 2 * vpt <= most && rows > kFewRows;
            if (more && threads > (backward || vpt > 1 ? 768 : 512)) continue;
            plan = {true, vpt, (int)threads, 0};
            break;
        }
    }
    if (backward) {
        const int waves = plan.block ? plan.threads / 64 : 4;
        const int64_t teams = plan.vpt == 0 || plan.block ? rows : (rows + 3) / 4;
        const int held = plan.vpt == 0 ? 2 : std::max(1, waves_held(plan.vpt * ne) / ((waves + 3) / 4));
        const int want = plan.block ? std::min(held, std::max(2, (16 + waves - 1) / waves)) : held;
        plan.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(256 * want, teams));
    }
    return plan;
}

hipError_t launch_norm(const swr_norm_t& n, const NormPlan& plan, const NormParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    if (n.dtype == SWR_DTYPE_F32) return forward<F32, F32>(n, plan, p, st);
    return n.weight_dtype == SWR_DTYPE_F32 ? forward<Bf16, F32>(n, plan, p, st) : forward<Bf16, Bf16>(n, plan, p, st);
}

hipError_t launch_norm_backward(const swr_norm_t& n, const NormPlan& plan, const NormParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    if (n.dtype == SWR_DTYPE_F32) return backward<F32, F32>(plan, p, st);
    return n.weight_dtype == SWR_DTYPE_F32 ? backward<Bf16, F32>(plan, p, st) : backward<Bf16, Bf16>(plan, p, st);
}

}  // namespace swr
