// swr_norm.hip -- residual addition and root-mean-square norm, forward and
// backward, on gfx950.
//
//     h = x + r;   y = h rho w,   rho = 1 / sqrt(mean(h^2) + eps)
//     n = h rho, g = dy w:   dx = rho (g - n mean(g n)) + dh,   dw = sum_rows dy n
//
// Every tensor is moved once: a row is held in registers between the sum over it
// and its outputs, by one wave (64 threads), four, or sixteen, with up to 32
// elements a thread.  The forward's two row sums (h^2 and, for 8-bit
// outputs, max|h w|) need the loads alone, so both are reduced together; so do
// the backward's (h^2 and g h).
#include <algorithm>

#include "swr_hybrid_launch.h"

namespace swr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of elements at any element's alignment: the hardware's wide loads
// and stores take unaligned addresses.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    u32x4 v;
};

// (By value: bit casts of a vector's element itself read its first.)
__device__ inline float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }

struct Bf16 {
    typedef uint16_t store;
    static constexpr int NE = 8;
    static __device__ float get(const u32x4& v, int i) {
        return as_float(i % 2 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
    }
    static __device__ float one(store s) { return __builtin_bit_cast(float, (uint32_t)s << 16); }
    static __device__ store to(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
    static __device__ u32x4 pack(const float* f) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (uint32_t)to(f[2 * i]) | (uint32_t)to(f[2 * i + 1]) << 16;
        return v;
    }
};
struct F32 {
    typedef float store;
    static constexpr int NE = 4;
    static __device__ float get(const u32x4& v, int i) { return as_float(v[i]); }
    static __device__ float one(store s) { return s; }
    static __device__ store to(float f) { return f; }
    static __device__ u32x4 pack(const float* f) {
        return u32x4{__builtin_bit_cast(uint32_t, f[0]), __builtin_bit_cast(uint32_t, f[1]),
                     __builtin_bit_cast(uint32_t, f[2]), __builtin_bit_cast(uint32_t, f[3])};
    }
};

// n elements (n <= 0: none) of E at p, as NE floats, zeros past n.
template <class E, int NE>
__device__ inline void load(const typename E::store* p, int n, float* f) {
    if (n >= NE) {
#pragma unroll
        for (int j = 0; j < NE; j += E::NE) {
            const u32x4 v = ((const Loose<typename E::store>*)(p + j))->v;
#pragma unroll
            for (int i = 0; i < E::NE; ++i) f[j + i] = E::get(v, i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) f[i] = i < n ? E::one(p[i]) : 0.0f;
    }
}

template <class E, int NE>
__device__ inline void store(typename E::store* p, int n, const float* f) {
    if (n >= NE) {
#pragma unroll
        for (int j = 0; j < NE; j += E::NE) ((Loose<typename E::store>*)(p + j))->v = E::pack(f + j);
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (i < n) p[i] = E::to(f[i]);
    }
}

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ inline uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

// Sums of a and b over the TPR threads of a row; every thread gets them, in
// the same order on every thread.  `buf` holds 2 values a wave of the block.
template <int TPR>
__device__ inline void row_sums(float& a, float& b, float* buf) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        const int wave = threadIdx.x / 64;
        __syncthreads();   // (the last row's values have been read)
        if (threadIdx.x % 64 == 0) { buf[2 * wave] = a; buf[2 * wave + 1] = b; }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < NW; ++i) { a += buf[2 * i]; b += buf[2 * i + 1]; }
    }
}
template <int TPR>
__device__ inline void row_sum_max(float& a, uint32_t& b, float* buf) {
    a = wave_sum(a);
    b = wave_max(b);
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        const int wave = threadIdx.x / 64;
        __syncthreads();
        if (threadIdx.x % 64 == 0) { buf[2 * wave] = a; buf[2 * wave + 1] = __builtin_bit_cast(float, b); }
        __syncthreads();
        a = 0.0f;
        b = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) { a += buf[2 * i]; b = max(b, __builtin_bit_cast(uint32_t, buf[2 * i + 1])); }
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
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (i < n) p[i] = (uint8_t)(w[i / 4] >> 8 * (i % 4));
    }
}

constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

template <class E, class WE, int TPR, int VPT, bool FP8>
__global__ __launch_bounds__(block_of(TPR)) void swr_norm_kernel(NormParams p) {
    constexpr int NE = E::NE, BLOCK = block_of(TPR);
    typedef typename E::store T;
    typedef typename WE::store WT;
    __shared__ float buf[2 * BLOCK / 64];
    const int t = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * (BLOCK / TPR) + threadIdx.x / TPR; row < p.rows;
         row += (int64_t)gridDim.x * (BLOCK / TPR)) {
        const T* x = (const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i);
        const T* r = p.r ? (const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i) : nullptr;
        float h[VPT][NE], w[VPT][NE];
#pragma unroll
        for (int v = 0; v < VPT; ++v) load<E, NE>(x + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, h[v]);
        if (r) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float f[NE];
                load<E, NE>(r + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, f);
#pragma unroll
                for (int i = 0; i < NE; ++i) h[v][i] += f[i];
            }
        }
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            load<WE, NE>((const WT*)p.w + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, w[v]);
        if (p.h) {
            T* ho = (T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i);
#pragma unroll
            for (int v = 0; v < VPT; ++v) store<E, NE>(ho + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, h[v]);
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
            row_sum_max<TPR>(sum, top, buf);
        } else {
            float none = 0.0f;
            row_sums<TPR>(sum, none, buf);
        }
        const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
        const int64_t yo = row_offset(row, p.inner, p.sy_o, p.sy_i);
        if constexpr (FP8) {
            const Codes code(__builtin_bit_cast(float, top) * rho);
            if (t == 0) p.scale[row] = code.scale;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float f[NE];
#pragma unroll
                for (int i = 0; i < NE; ++i) f[i] = code(h[v][i] * w[v][i] * rho);
                store_codes<NE>((uint8_t*)p.y + yo + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, f);
            }
        } else {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float f[NE];
#pragma unroll
                for (int i = 0; i < NE; ++i) f[i] = h[v][i] * rho * w[v][i];
                store<E, NE>((T*)p.y + yo + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, f);
            }
        }
    }
}

// Rows too wide for registers: 1024 threads walk a row twice, the second time
// out of the L2 or the 256 MB cache.  h is stored on the second walk, by the
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
            const int n = p.width - (int)e;
            float h[NE], f[NE];
            load<E, NE>(x + e, n, h);
            if (r) {
                load<E, NE>(r + e, n, f);
#pragma unroll
                for (int i = 0; i < NE; ++i) h[i] += f[i];
            }
            if constexpr (FP8) load<WE, NE>((const WT*)p.w + e, n, f);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                sum += h[i] * h[i];
                if constexpr (FP8) top = max(top, __builtin_bit_cast(uint32_t, h[i] * f[i]) & 0x7fffffffu);
            }
        }
        row_sum_max<1024>(sum, top, buf);
        const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
        const Codes code(__builtin_bit_cast(float, top) * rho);
        if constexpr (FP8)
            if (threadIdx.x == 0) p.scale[row] = code.scale;
        T* ho = p.h ? (T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i) : nullptr;
        const int64_t yo = row_offset(row, p.inner, p.sy_o, p.sy_i);
        for (int64_t e = (int64_t)threadIdx.x * NE; e < p.width; e += 1024 * NE) {
            const int n = p.width - (int)e;
            float h[NE], f[NE];
            load<E, NE>(x + e, n, h);
            if (r) {
                load<E, NE>(r + e, n, f);
#pragma unroll
                for (int i = 0; i < NE; ++i) h[i] += f[i];
            }
            if (ho) store<E, NE>(ho + e, n, h);
            load<WE, NE>((const WT*)p.w + e, n, f);
#pragma unroll
            for (int i = 0; i < NE; ++i) f[i] = FP8 ? code(h[i] * f[i] * rho) : h[i] * rho * f[i];
            if constexpr (FP8) store_codes<NE>((uint8_t*)p.y + yo + e, n, f);
            else store<E, NE>((T*)p.y + yo + e, n, f);
        }
    }
}

// Backward.  A row's TPR threads take rows in turn and keep their columns'
// shares of dw in registers; a block joins its rows' shares in LDS, in order,
// and writes one row of `partial`, which swr_norm_dw_kernel sums.
template <class E, class WE, int TPR, int VPT>
__global__ __launch_bounds__(block_of(TPR)) void swr_norm_bwd_kernel(NormParams p) {
    constexpr int NE = E::NE, BLOCK = block_of(TPR), RPB = BLOCK / TPR;
    typedef typename E::store T;
    typedef typename WE::store WT;
    __shared__ float buf[2 * BLOCK / 64];
    __shared__ float share[RPB > 1 ? TPR * VPT * NE : 1];
    const int t = threadIdx.x % TPR;
    float dw[VPT][NE] = {};
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        const T* hr = (const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i);
        const T* dy = (const T*)p.y + row_offset(row, p.inner, p.sy_o, p.sy_i);
        const T* dh = p.r ? (const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i) : nullptr;
        float h[VPT][NE], g[VPT][NE], d[VPT][NE];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * NE, n = p.width - e;
            load<E, NE>(hr + e, n, h[v]);
            load<E, NE>(dy + e, n, d[v]);
        }
        float sum = 0.0f, along = 0.0f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float w[NE];
            load<WE, NE>((const WT*)p.w + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, w);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                g[v][i] = d[v][i] * w[i];
                sum += h[v][i] * h[v][i];
                along += g[v][i] * h[v][i];
            }
        }
        row_sums<TPR>(sum, along, buf);
        const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
        const float c = along / (float)p.width * rho * rho;   // mean(g n) rho, times h: n mean(g n)
        T* dx = (T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * NE, n = p.width - e;
            float f[NE] = {};
            if (dh) load<E, NE>(dh + e, n, f);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                f[i] += rho * (g[v][i] - h[v][i] * c);
                dw[v][i] += d[v][i] * (h[v][i] * rho);
            }
            store<E, NE>(dx + e, n, f);
        }
    }
    float* out = p.partial + (int64_t)blockIdx.x * p.width;
    if constexpr (RPB > 1) {
#pragma unroll 1
        for (int k = 0; k < RPB; ++k) {
            __syncthreads();
            if ((int)threadIdx.x / TPR == k) {
#pragma unroll
                for (int v = 0; v < VPT; ++v)
#pragma unroll
                    for (int i = 0; i < NE; ++i) {
                        float* s = share + (v * NE + i) * TPR + t;
                        if (k > 0) dw[v][i] += *s;
                        *s = dw[v][i];
                    }
            }
        }
    }
    if (RPB == 1 || (int)threadIdx.x / TPR == RPB - 1) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) store<F32, NE>(out + (v * TPR + t) * NE, p.width - (v * TPR + t) * NE, dw[v]);
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
            const int n = p.width - (int)e;
            float h[NE], d[NE], w[NE];
            load<E, NE>(hr + e, n, h);
            load<E, NE>(dy + e, n, d);
            load<WE, NE>((const WT*)p.w + e, n, w);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                sum += h[i] * h[i];
                along += d[i] * w[i] * h[i];
            }
        }
        row_sums<1024>(sum, along, buf);
        if (threadIdx.x == 0) {
            const float rho = 1.0f / sqrtf(sum / (float)p.width + p.eps);
            p.stats[row] = make_float2(rho, along / (float)p.width * rho * rho);
        }
    }
}

// Second walk: a block takes 256 vectors of columns (blockIdx.y) of every
// gridDim.x-th row.
template <class E, class WE>
__global__ __launch_bounds__(256) void swr_norm_bwd_wide_kernel(NormParams p) {
    constexpr int NE = E::NE;
    typedef typename E::store T;
    typedef typename WE::store WT;
    const int64_t e = ((int64_t)blockIdx.y * 256 + threadIdx.x) * NE;
    if (e >= p.width) return;
    const int n = p.width - (int)e;
    float w[NE], dw[NE] = {};
    load<WE, NE>((const WT*)p.w + e, n, w);
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const float2 s = p.stats[row];
        float h[NE], d[NE], f[NE] = {};
        load<E, NE>((const T*)p.x + row_offset(row, p.inner, p.sx_o, p.sx_i) + e, n, h);
        load<E, NE>((const T*)p.y + row_offset(row, p.inner, p.sy_o, p.sy_i) + e, n, d);
        if (p.r) load<E, NE>((const T*)p.r + row_offset(row, p.inner, p.sr_o, p.sr_i) + e, n, f);
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            f[i] += s.x * (d[i] * w[i] - h[i] * s.y);
            dw[i] += d[i] * (h[i] * s.x);
        }
        store<E, NE>((T*)p.h + row_offset(row, p.inner, p.sh_o, p.sh_i) + e, n, f);
    }
    store<F32, NE>(p.partial + (int64_t)blockIdx.x * p.width + e, n, dw);
}

// dw: the sum of `blocks` rows of partial, 64 columns a block, its 16 waves
// each taking every 16th row, then joined in order.
__global__ __launch_bounds__(1024) void swr_norm_dw_kernel(const float* partial, float* dw, int width, int blocks) {
    __shared__ float buf[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (col < width)
        for (int b = wave; b < blocks; b += 16) s += partial[(int64_t)b * width + col];
    buf[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < width) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += buf[i][lane];
        dw[col] = s;
    }
}

// Most floats of a row that a thread holds: 32 with one or four waves a row,
// which leaves the forward's x, r and w and the backward's h, g, dy and dw
// room in 256 registers; with sixteen waves (128 registers) 32 in the
// forward and 16 in the backward.
constexpr int kHeld = 32, kHeldWide = 16;
constexpr int kDwBlocks = 512;   // backward: two blocks a compute unit
constexpr int64_t kMostBlocks = 1 << 20;   // of a forward launch, whose blocks take rows in turn

unsigned grid_of(int64_t blocks) { return (unsigned)std::min(blocks, kMostBlocks); }

template <class F>
hipError_t by_plan(const NormPlan& plan, F f) {
    switch (plan.tpr * 16 + plan.vpt) {
        case 64 * 16 + 1: return f.template operator()<64, 1>();
        case 64 * 16 + 2: return f.template operator()<64, 2>();
        case 64 * 16 + 4: return f.template operator()<64, 4>();
        case 64 * 16 + 8: return f.template operator()<64, 8>();
        case 256 * 16 + 1: return f.template operator()<256, 1>();
        case 256 * 16 + 2: return f.template operator()<256, 2>();
        case 256 * 16 + 4: return f.template operator()<256, 4>();
        case 256 * 16 + 8: return f.template operator()<256, 8>();
        case 1024 * 16 + 1: return f.template operator()<1024, 1>();
        case 1024 * 16 + 2: return f.template operator()<1024, 2>();
        case 1024 * 16 + 4: return f.template operator()<1024, 4>();
        case 1024 * 16 + 8: return f.template operator()<1024, 8>();
        default: return hipErrorInvalidValue;
    }
}

template <class E, class WE, bool FP8>
struct Forward {
    const NormParams& p;
    hipStream_t st;
    template <int TPR, int VPT>
    hipError_t operator()() const {
        if constexpr (VPT * E::NE <= kHeld) {
            constexpr int RPB = block_of(TPR) / TPR;
            hipLaunchKernelGGL((swr_norm_kernel<E, WE, TPR, VPT, FP8>), dim3(grid_of((p.rows + RPB - 1) / RPB)),
                               dim3(block_of(TPR)), 0, st, p);
            return hipGetLastError();
        } else {
            return hipErrorInvalidValue;
        }
    }
};

template <class E, class WE>
struct Backward {
    const NormParams& p;
    hipStream_t st;
    int blocks;
    template <int TPR, int VPT>
    hipError_t operator()() const {
        if constexpr (VPT * E::NE <= (TPR > 256 ? kHeldWide : kHeld)) {
            hipLaunchKernelGGL((swr_norm_bwd_kernel<E, WE, TPR, VPT>), dim3((unsigned)blocks), dim3(block_of(TPR)), 0,
                               st, p);
            return hipGetLastError();
        } else {
            return hipErrorInvalidValue;
        }
    }
};

template <class E, class WE>
hipError_t forward(const swr_norm_t& n, const NormPlan& plan, const NormParams& p, hipStream_t st) {
    const bool fp8 = n.out_dtype == SWR_DTYPE_FP8;
    if (plan.vpt == 0) {
        if (fp8) hipLaunchKernelGGL((swr_norm_wide_kernel<E, WE, true>), dim3(grid_of(p.rows)), dim3(1024), 0, st, p);
        else hipLaunchKernelGGL((swr_norm_wide_kernel<E, WE, false>), dim3(grid_of(p.rows)), dim3(1024), 0, st, p);
        return hipGetLastError();
    }
    return fp8 ? by_plan(plan, Forward<E, WE, true>{p, st}) : by_plan(plan, Forward<E, WE, false>{p, st});
}

template <class E, class WE>
hipError_t backward(const NormPlan& plan, const NormParams& p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (p.rows == 0) {
        // (dw is a sum of nothing)
    } else if (plan.vpt == 0) {
        hipLaunchKernelGGL((swr_norm_stats_kernel<E, WE>), dim3(grid_of(p.rows)), dim3(1024), 0, st, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const unsigned cols = (unsigned)((p.width + 256 * E::NE - 1) / (256 * E::NE));
        hipLaunchKernelGGL((swr_norm_bwd_wide_kernel<E, WE>), dim3((unsigned)plan.blocks, cols), dim3(256), 0, st, p);
        e = hipGetLastError();
    } else {
        e = by_plan(plan, Backward<E, WE>{p, st, plan.blocks});
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(swr_norm_dw_kernel, dim3((unsigned)((p.width + 63) / 64)), dim3(1024), 0, st, p.partial, p.dw,
                       p.width, plan.blocks);
    return hipGetLastError();
}

}  // namespace

NormPlan plan_norm(int dtype, int64_t rows, int64_t width, bool backward) {
    const int ne = dtype == SWR_DTYPE_BF16 ? Bf16::NE : F32::NE;
    const int64_t vectors = (width + ne - 1) / ne;
    NormPlan plan{0, 0, 0};
    for (int tpr : {64, 256, 1024}) {
        const int most = (tpr > 256 && backward ? kHeldWide : kHeld) / ne;
        if (vectors > (int64_t)most * tpr) continue;
        plan.tpr = tpr;
        for (plan.vpt = 1; (int64_t)plan.vpt * tpr < vectors;) plan.vpt *= 2;
        break;
    }
    if (backward) {
        const int64_t per = plan.vpt == 0 ? 1 : plan.tpr < 256 ? 256 / plan.tpr : 1;
        plan.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(kDwBlocks, (rows + per - 1) / per));
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
