// swr_fp4.hip -- products of a few rows with 4-bit weights, on gfx950.
//
//     y[m, n] = s[m] sum_k x[m, k] value(code[n, k]) 2^(power[n, k / 32] - 127)
//
// A wave takes 16 rows of W (R tiles of them) and 16 rows of x (MT tiles) over
// its share of k; the block's waves share out k, and join in LDS.  W is the
// matrix instructions' A operand, so that a lane holds 32 weights of one row in
// 16 bytes, with their one power:
//   * 8-bit x: the scaled matrix instruction takes codes and powers as they lie.
//     Its sums of 128 products are off by up to 1.2e-5 of the sum of their absolute
//     values (measured; the bf16 instruction's by 2^-24 of it), far below the
//     rounding of a bf16 y, 2^-9; for a float32 y, x becomes bf16, exactly, and goes as below;
//   * bf16 x: the conversion instruction makes bf16 pairs of code times power, exactly;
//   * float32 x: the same against x split into three bf16 parts, which hold all
//     of its 24 bits.
// What bounds it is the weights' bytes: 17 a group of 32, read once for 64 rows
// of x.
#include <algorithm>

#include "swr_hybrid_launch.h"

namespace swr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    u32x4 v;
};

// 16 bytes of row elements at p, of which n elements (n <= 0: none) exist;
// zeros past them.
template <class T>
__device__ inline u32x4 load16(const T* p, int n) {
    constexpr int NE = 16 / sizeof(T);
    if (n >= NE) return ((const Loose<T>*)p)->v;
    T e[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) e[i] = i < n ? p[i] : T(0);
    return __builtin_bit_cast(u32x4, e);
}

// (By value: a bit cast of a vector's element itself reads its first.)
__device__ inline float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }

struct XBf16 {
    typedef uint16_t T;
    static constexpr int kParts = 1;
};
struct XF32 {
    typedef float T;
    static constexpr int kParts = 3;
};
struct XFp8 {          // for a bf16 y
    typedef uint8_t T;
};
struct XFp8Exact {     // for a float32 y
    typedef uint8_t T;
    static constexpr int kParts = 1;
};

// A lane's x operands of one block of 128 k.
template <class X>
struct Fragment;

template <>
struct Fragment<XBf16> {
    bf16x8 v[4][1];   // matrix instruction j: k = 32 q + 8 j ...
    __device__ void load(const uint16_t* row, int k0, int q, int K) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = k0 + 32 * q + 8 * j;
            v[j][0] = __builtin_bit_cast(bf16x8, load16(row + k, K - k));
        }
    }
};

template <>
struct Fragment<XF32> {
    bf16x8 v[4][3];
    __device__ void load(const float* row, int k0, int q, int K) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 32 * q + 8 * j + 4 * h;
                const u32x4 u = load16(row + k, K - k);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // Cut off, not rounded: nothing overflows, and each part
                    // has 8 of the 24 bits.  An infinity or a NaN is all in the first.
                    const float f = as_float(u[i]);
                    const bool finite = (u[i] & 0x7f800000u) != 0x7f800000u;
                    const uint32_t a = f != f ? 0x7fc00000u : u[i] & 0xffff0000u;
                    const float r = finite ? f - as_float(a) : 0.0f;
                    const uint32_t b = __builtin_bit_cast(uint32_t, r) & 0xffff0000u;
                    const float s = r - as_float(b);
                    v[j][0][4 * h + i] = __builtin_bit_cast(__bf16, (uint16_t)(a >> 16));
                    v[j][1][4 * h + i] = __builtin_bit_cast(__bf16, (uint16_t)(b >> 16));
                    v[j][2][4 * h + i] = (__bf16)s;
                }
            }
        }
    }
};

template <>
struct Fragment<XFp8Exact> {
    bf16x8 v[4][1];
    __device__ void load(const uint8_t* row, int k0, int q, int K) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + 32 * q + 16 * h;
            const u32x4 u = load16(row + k, K - k);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], 1.0f, false);
                const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], 1.0f, true);
                bf16x8& w = v[2 * h + i / 2][0];
                w[i % 2 * 4] = a[0]; w[i % 2 * 4 + 1] = a[1]; w[i % 2 * 4 + 2] = b[0]; w[i % 2 * 4 + 3] = b[1];
            }
        }
    }
};

template <>
struct Fragment<XFp8> {
    u32x4 v[2];   // the scaled instruction's 8-bit operand: k = 16 q ... and 64 + 16 q ...
    __device__ void load(const uint8_t* row, int k0, int q, int K) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + 64 * h + 16 * q;
            v[h] = load16(row + k, K - k);
        }
    }
};

template <int PART>
__device__ inline bf16x2 pair_of(uint32_t codes, float power) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, PART);
}

// acc += W x over 128 k: codes (32 of the lane's row, from k0 + 32 q) and
// their power against MT tiles' fragments.
template <class X, int MT>
__device__ inline void multiply(const u32x4& codes, uint32_t power, const Fragment<X> (&x)[MT], f32x4 (&acc)[MT]) {
    // 2^(power - 127); 0 stands for 2^-127 (below the normal floats), 255 for NaN
    const float scale = __builtin_bit_cast(float, power == 255 ? 0x7fc00000u : power ? power << 23 : 0x00400000u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bf16x2 p0 = pair_of<0>(codes[j], scale), p1 = pair_of<1>(codes[j], scale);
        const bf16x2 p2 = pair_of<2>(codes[j], scale), p3 = pair_of<3>(codes[j], scale);
        const bf16x8 w{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int c = 0; c < X::kParts; ++c)
                acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[m].v[j][c], acc[m], 0, 0, 0);
    }
}
template <int MT>
__device__ inline void multiply(const u32x4& codes, uint32_t power, const Fragment<XFp8> (&x)[MT], f32x4 (&acc)[MT]) {
    const i32x8 w{(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const i32x8 b{(int)x[m].v[0][0], (int)x[m].v[0][1], (int)x[m].v[0][2], (int)x[m].v[0][3],
                      (int)x[m].v[1][0], (int)x[m].v[1][1], (int)x[m].v[1][2], (int)x[m].v[1][3]};
        acc[m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, b, acc[m], 4 /* codes */, 0 /* e4m3 */, 0,
                                                                (int)power, 0, 127);
    }
}

template <class Y>
__device__ inline void put(Y* p, float f);
template <>
__device__ inline void put<float>(float* p, float f) { *p = f; }
template <>
__device__ inline void put<uint16_t>(uint16_t* p, float f) { *p = __builtin_bit_cast(uint16_t, (__bf16)f); }

constexpr int kWaves = 8;

template <class X, class Y, int R, int MT>
__global__ __launch_bounds__(kWaves * 64) void swr_fp4_kernel(Fp4Params p) {
    typedef typename X::T T;
    __shared__ f32x4 join[kWaves][R * MT][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 16, q = lane / 16;
    const int n0 = (int)blockIdx.x * 16 * R;
    const int m0 = (int)blockIdx.y * 16 * MT;
    f32x4 acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[r][m] = f32x4{0, 0, 0, 0};
    const int groups = (p.K + 31) / 32, blocks = (groups + 3) / 4;
    for (int kb = wave; kb < blocks; kb += kWaves) {
        const int group = kb * 4 + q;
        u32x4 codes[R];
        uint32_t power[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = n0 + 16 * r + l;
            codes[r] = u32x4{0, 0, 0, 0};
            power[r] = 127;
            if (n < p.N && group < groups) {
                codes[r] = *(const u32x4*)(p.codes + n * p.sc + group * 16);
                power[r] = p.powers[n * p.sp + group];
            }
        }
        Fragment<X> x[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = m0 + 16 * m + l;
            x[m].load((const T*)p.x + (row < p.M ? row : 0) * p.sx, kb * 128, q, row < p.M ? p.K : 0);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) multiply(codes[r], power[r], x, acc[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) join[wave][r * MT + m][lane] = acc[r][m];
    __syncthreads();
    // Tile t's sums, by the wave t % kWaves: the lane has rows 4 q ... of W and row l of x.
    for (int t = wave; t < R * MT; t += kWaves) {
        f32x4 sum = join[0][t][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += join[w][t][lane];
        const int row = m0 + t % MT * 16 + l, n = n0 + t / MT * 16 + 4 * q;
        if (row >= p.M) continue;
        const float s = p.scale ? p.scale[row] : 1.0f;
        Y* y = (Y*)p.y + row * p.sy + n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) put(y + i, sum[i] * s);
    }
}

// Codes of w: a lane takes a pair of weights, 16 lanes a group.
template <class T>
__global__ __launch_bounds__(256) void swr_fp4_pack_kernel(const T* w, int64_t N, int64_t K, int64_t sw,
                                                           uint8_t* codes, uint8_t* powers, int64_t sc, int64_t sp) {
    const int64_t groups = (K + 31) / 32, total = N * groups * 16;
    const int64_t whole = (total + 63) / 64 * 64;   // (every lane of a wave takes part in the groups' maxima)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < whole; i += (int64_t)gridDim.x * 256) {
        const bool in = i < total;
        const int64_t group = in ? i / 16 : 0, n = group / groups, g = group % groups, k = g * 32 + i % 16 * 2;
        float f[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f[j] = 0.0f;
            if (in && k + j < K) {
                if constexpr (sizeof(T) == 2) f[j] = __builtin_bit_cast(float, (uint32_t)w[n * sw + k + j] << 16);
                else f[j] = w[n * sw + k + j];
            }
        }
        uint32_t top = max(__builtin_bit_cast(uint32_t, f[0]) & 0x7fffffffu,
                           __builtin_bit_cast(uint32_t, f[1]) & 0x7fffffffu);
#pragma unroll
        for (int m = 8; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        if (!in) continue;
        // The least power with top <= 6 * 2^(power - 127): top's own exponent
        // less 2, and one more where its mantissa is over 1.5.
        int power = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u);
        power = top == 0 ? 127 : min(max(power, 1), 252);
        if (top >= 0x7f800000u) power = 255;
        const float scale = power == 255 ? 1.0f : __builtin_bit_cast(float, (uint32_t)power << 23);
        const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0], f[1], scale, 0);
        codes[n * sc + g * 16 + i % 16] = (uint8_t)c;
        if (i % 16 == 0) powers[n * sp + g] = (uint8_t)power;
    }
}

template <class X, class Y, int R, int MT>
hipError_t go(const Fp4Params& p, hipStream_t st) {
    const dim3 grid((unsigned)((p.N + 16 * R - 1) / (16 * R)), (unsigned)((p.M + 16 * MT - 1) / (16 * MT)));
    hipLaunchKernelGGL((swr_fp4_kernel<X, Y, R, MT>), grid, dim3(kWaves * 64), 0, st, p);
    return hipGetLastError();
}

template <class X, class Y>
hipError_t by_rows(const Fp4Params& p, hipStream_t st) {
    if (p.M <= 16) return go<X, Y, 1, 1>(p, st);
    if (p.M <= 32) return go<X, Y, 1, 2>(p, st);
    return go<X, Y, 1, 4>(p, st);
}

}  // namespace

hipError_t launch_fp4(int dtype, int out_dtype, const Fp4Params& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    const bool f32 = out_dtype == SWR_DTYPE_F32;
    if (dtype == SWR_DTYPE_FP8) return f32 ? by_rows<XFp8Exact, float>(p, st) : by_rows<XFp8, uint16_t>(p, st);
    if (dtype == SWR_DTYPE_BF16) return f32 ? by_rows<XBf16, float>(p, st) : by_rows<XBf16, uint16_t>(p, st);
    return f32 ? by_rows<XF32, float>(p, st) : by_rows<XF32, uint16_t>(p, st);
}

hipError_t launch_fp4_pack(int dtype, const void* w, int64_t N, int64_t K, int64_t sw, uint8_t* codes, uint8_t* powers,
                           int64_t sc, int64_t sp, void* stream) {
    const int64_t total = N * ((K + 31) / 32) * 16;
    const dim3 grid((unsigned)std::min<int64_t>((total + 255) / 256, 1 << 16));
    if (dtype == SWR_DTYPE_BF16)
        hipLaunchKernelGGL((swr_fp4_pack_kernel<uint16_t>), grid, dim3(256), 0, (hipStream_t)stream,
                           (const uint16_t*)w, N, K, sw, codes, powers, sc, sp);
    else
        hipLaunchKernelGGL((swr_fp4_pack_kernel<float>), grid, dim3(256), 0, (hipStream_t)stream, (const float*)w, N,
                           K, sw, codes, powers, sc, sp);
    return hipGetLastError();
}

}  // namespace swr
