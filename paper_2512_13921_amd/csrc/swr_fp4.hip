// swr_fp4.hip -- products of a few rows with 4-bit weights, on gfx950.
//
//     y[m, n] = s[m] sum_k x[m, k] value(code[n, k]) 2^(power[n, k / 32] - 127)
//
// A wave takes tiles of 16 rows of W (R) and of x (MT) over its share of k; the
// block's waves share out k, and join in LDS.  One kernel loads x along with W, the
// other holds its share of x in registers and goes over W.  W is the matrix
// instructions' A operand, so that a lane holds 32 weights of one row in 16 bytes, with
// their one power:
//   * bf16 x: the conversion instruction makes bf16 pairs of code times power, exactly;
//   * 8-bit x: the same against x made bf16, exactly.  (The matrix instruction that takes
//     codes, powers and 8-bit values as they lie would save the conversions, 31.3 us for 32.9
//     below, and 20 for 28 where x does not stay in registers, 16 x 16384 to 8192; but its sums
//     of 128 products are off by up to 1.2e-5 of the sum of their
//     absolute values, which shows in a bf16 y where they cancel);
//   * float32 x: the same against x split into three bf16 parts, which hold all
//     of its 24 bits.
// What bounds it is the weights' bytes, 17 a group of 32: 16 x 8192 8-bit rows
// against 28672 take 33 us, 3.8 TB/s, where a copy reaches 5.2 and a loop over codes
// and powers alone 5.0; against twice as many 61, so that 28 us are the tiles (4.4 TB/s) and 5
// what is before them, the launch and x, which all CUs load first.  Few or short rows are bound
// by latency: 2048 to 6176 for one token 4.7 us.  float32 is bound by its conversion, anew for
// every tile where x does not stay in registers (past 2048), and three products.
#include <algorithm>
#include <type_traits>

#include "swr_hybrid_launch.h"

namespace swr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    u32x4 v;
};

// How 16 bytes of a row of K elements are loaded from element k on, zeros past K:
// kWhole where all are there; kEven where K is a multiple of 16 bytes' elements, by an
// unconditional load and a selection, so that loads follow each other without
// branches; kAny in branches, element by element at the end.
enum Ends { kWhole, kEven, kAny };
template <Ends ENDS, class T>
__device__ inline u32x4 load16(const T* row, int k, int K) {
    constexpr int NE = 16 / sizeof(T);
    if constexpr (ENDS == kWhole) return ((const Loose<T>*)(row + k))->v;
    if constexpr (ENDS == kEven) {
        const u32x4 v = ((const Loose<T>*)(row + min(k, K - NE)))->v;
        const u32x4 none{0, 0, 0, 0};
        return k < K ? v : none;
    }
    if (k + NE <= K) return ((const Loose<T>*)(row + k))->v;
    T e[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) e[i] = k + i < K ? row[k + i] : T(0);
    return __builtin_bit_cast(u32x4, e);
}

// (By value: a bit cast of a vector's element itself reads its first.)
__device__ inline float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }

struct XBf16 {
    static constexpr bool kStaged = true;
    typedef uint16_t T;
    static constexpr int kParts = 1;
};
struct XF32 {
    static constexpr bool kStaged = false;
    typedef float T;
    static constexpr int kParts = 3;
};
struct XFp8 {
    static constexpr bool kStaged = true;
    typedef uint8_t T;
    static constexpr int kParts = 1;
};

// A lane's x operands against 32 weights of each quarter q, of group `of(q)` of 32 k.
template <class X>
struct Fragment;

template <>
struct Fragment<XBf16> {
    static constexpr int kVectors = 4;
    bf16x8 v[4][1];   // matrix instruction j: the group's k = 8 j ...
    __device__ void put(int i, const u32x4& u) { v[i][0] = __builtin_bit_cast(bf16x8, u); }
    __device__ u32x4 get(int i) const { return __builtin_bit_cast(u32x4, v[i][0]); }
    __device__ bf16x8 part(int j, int) const { return v[j][0]; }
    // Where vector i is, in elements from the block's first: group g of quarter q's G.
    static __device__ int at(int i, int q, int g, int G) { return 32 * (q * G + g) + 8 * i; }
    template <Ends ENDS, class Of>
    __device__ void load(const uint16_t* row, Of of, int q, int K) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = 32 * of(q) + 8 * j;
            v[j][0] = __builtin_bit_cast(bf16x8, load16<ENDS>(row, k, K));
        }
    }
};

template <>
struct Fragment<XF32> {
    bf16x8 v[4][3];
    __device__ bf16x8 part(int j, int c) const { return v[j][c]; }
    template <Ends ENDS, class Of>
    __device__ void load(const float* row, Of of, int q, int K) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = 32 * of(q) + 8 * j + 4 * h;
                const u32x4 u = load16<ENDS>(row, k, K);
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

// (Kept as they are, and made bf16, exactly, for each product: half the registers.)
template <>
struct Fragment<XFp8> {
    static constexpr int kVectors = 2;
    u32x4 v[2];
    __device__ void put(int i, const u32x4& u) { v[i] = u; }
    __device__ u32x4 get(int i) const { return v[i]; }
    static __device__ int at(int i, int q, int g, int G) { return 32 * (q * G + g) + 16 * i; }
    // Hides from the compiler that the values are the last tile's still, as it would convert
    // them once for all: faster where that fits (64 x 4096 to 4096 9.0 us, 9.4 hidden), and
    // spilled where not (64 x 8192 to 28672 250 us, 69 hidden).
    __device__ void hide() { asm volatile("" : "+v"(v[0]), "+v"(v[1])); }
    __device__ bf16x8 part(int j, int) const {
        const uint32_t lo = v[j / 2][j % 2 * 2], hi = v[j / 2][j % 2 * 2 + 1];
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    template <Ends ENDS, class Of>
    __device__ void load(const uint8_t* row, Of of, int q, int K) {
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = load16<ENDS>(row, 32 * of(q) + 16 * h, K);
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
                acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[m].part(j, c), acc[m], 0, 0, 0);
    }
}
template <class Y>
__device__ inline void put(Y* p, float f);
template <>
__device__ inline void put<float>(float* p, float f) { *p = f; }
template <>
__device__ inline void put<uint16_t>(uint16_t* p, float f) { *p = __builtin_bit_cast(uint16_t, (__bf16)f); }

constexpr int kWaves = 8;
constexpr int kCus = 256;

// One block of 128 G k of a wave's R tiles of W and MT tiles of x.  A lane takes G
// groups of a row that lie next to each other, 16 G bytes of codes.
template <class X, int R, int MT, int G>
struct Step {
    u32x4 codes[G][R];
    uint32_t power[G][R];
    Fragment<X> x[G][MT];
    // Rows past N or M are the last ones again (their sums are not stored).
    template <Ends ENDS>
    __device__ void load(const Fp4Params& p, const int (&n)[R], const int (&m)[MT], int kb, int q) {
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const auto of = [&](int quarter) { return (kb * 4 + quarter) * G + j; };
            const int group = of(q);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool in = ENDS == kWhole || group < (p.K + 31) / 32;
                codes[j][r] = in ? *(const u32x4*)(p.codes + n[r] * p.sc + group * 16) : u32x4{0, 0, 0, 0};
                power[j][r] = in ? p.powers[n[r] * p.sp + group] : 127;
            }
#pragma unroll
            for (int t = 0; t < MT; ++t)
                x[j][t].template load<ENDS>((const typename X::T*)p.x + m[t] * p.sx, of, q, p.K);
        }
    }
    __device__ void multiply_into(f32x4 (&acc)[R][MT]) const {
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
            for (int r = 0; r < R; ++r) multiply(codes[j][r], power[j][r], x[j], acc[r]);
    }
};

// A block's 8 waves are WK along k times 8 / WK along the rows of W; those along
// k take its blocks in turn and are joined in LDS, those along W read the same
// x at about the same time, mostly from the L1.  AHEAD blocks' loads are on their
// way at once.
template <class X, class Y, int R, int MT, int G, int WK, int AHEAD>
__global__ __launch_bounds__(kWaves * 64) void swr_fp4_kernel(Fp4Params p) {
    constexpr int WN = kWaves / WK;
    __shared__ f32x4 join[WK > 1 ? kWaves : 1][R * MT][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 16, q = lane / 16;
    const int wn = wave % WN, wk = wave / WN;
    const int n0 = (int)(blockIdx.x / p.m_blocks) * 16 * R * WN + wn * 16 * R;
    const int m0 = (int)(blockIdx.x % p.m_blocks) * 16 * MT;
    int n[R], m[MT];
#pragma unroll
    for (int r = 0; r < R; ++r) n[r] = min(n0 + 16 * r + l, p.N - 1);
#pragma unroll
    for (int t = 0; t < MT; ++t) m[t] = min(m0 + 16 * t + l, p.M - 1);
    f32x4 acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[r][t] = f32x4{0, 0, 0, 0};
    const int whole = p.K / (128 * G);
    int kb = wk;
    for (; kb + (AHEAD - 1) * WK < whole; kb += AHEAD * WK) {
        Step<X, R, MT, G> s[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) s[a].template load<kWhole>(p, n, m, kb + a * WK, q);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) s[a].multiply_into(acc);
    }
    for (; kb < whole; kb += WK) {
        Step<X, R, MT, G> s;
        s.template load<kWhole>(p, n, m, kb, q);
        s.multiply_into(acc);
    }
    if (kb == whole && p.K % (128 * G)) {
        Step<X, R, MT, G> s;
        s.template load<kAny>(p, n, m, kb, q);
        s.multiply_into(acc);
    }
    if constexpr (WK > 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < MT; ++t) join[wave][r * MT + t][lane] = acc[r][t];
        __syncthreads();
    }
    // Tile t's sums, by the wave along k that has its turn: the lane has rows 4 q
    // ... of W and row l of x.
#pragma unroll
    for (int t = 0; t < R * MT; ++t) {
        if (t % WK != wk) continue;
        f32x4 sum = acc[t / MT][t % MT];
        if constexpr (WK > 1) {
            sum = join[wn][t][lane];
#pragma unroll
            for (int w = 1; w < WK; ++w) sum += join[w * WN + wn][t][lane];
        }
        const int row = m0 + t % MT * 16 + l, col = n0 + t / MT * 16 + 4 * q;
        if (row >= p.M) continue;
        const float f = p.scale ? p.scale[row] : 1.0f;
        Y* y = (Y*)p.y + row * p.sy + col;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < p.N) put(y + i, sum[i] * f);
    }
}

// Registers that a lane holds x in, and the most that it may.
template <class X, int MT, int NB>
constexpr int held() {
    return (int)sizeof(Fragment<X>) / 4 * MT * NB;
}
constexpr int kMostHeld = 128;
// Whether 8-bit x, made bf16, would not fit.
template <class X, int MT, int NB>
constexpr bool kHidden = std::is_same<X, XFp8>::value && 2 * held<X, MT, NB>() > kMostHeld;

// The same with x in registers: a block's 8 waves share out k, each keeps what it
// needs of x (NB blocks of 128 k) and takes the tiles of 16 rows of W in turn with the
// other blocks, the next tile's codes on their way while one is worked on.
template <class X, int NB>
struct Codes {
    static constexpr int G = NB > 1 ? 2 : 1;
    u32x4 codes[NB];
    uint32_t power[NB / G];
    // Groups past the row's last, of which x is zeros, are the last again.
    __device__ void load(const Fp4Params& p, int tile, int wave, int l, int q) {
        const int n = min(tile * 16 + l, p.N - 1), last = (p.K + 31) / 32 - 1;
        const uint8_t* row = p.codes + n * p.sc;
        const uint8_t* powers = p.powers + n * p.sp;
#pragma unroll
        for (int j = 0; j < NB / G; ++j) {
            const int group = ((j * kWaves + wave) * 4 + q) * G;
            if constexpr (G == 2) {
                const int g = min(group, last), h = min(group + 1, last);
                codes[2 * j] = *(const u32x4*)(row + g * 16);
                codes[2 * j + 1] = *(const u32x4*)(row + h * 16);
                power[j] = powers[g] | (uint32_t)powers[h] << 8;
            } else {
                const int g = min(group, last);
                codes[j] = *(const u32x4*)(row + g * 16);
                power[j] = powers[g];
            }
        }
    }
};

template <class X, class Y, int MT, int NB, int DEPTH>
__global__ __launch_bounds__(kWaves * 64) void swr_fp4_held_kernel(Fp4Params p) {
    constexpr int G = Codes<X, NB>::G, TURNS = 4 / MT;
    __shared__ f32x4 join[2][TURNS][kWaves][MT][64];
    __shared__ u32x4 stage[X::kStaged ? kWaves : 1][X::kStaged ? 16 * (8 * G * (int)sizeof(typename X::T) + 1) : 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 16, q = lane / 16;
    const int m0 = (int)(blockIdx.x % p.m_blocks) * 16 * MT, first = (int)(blockIdx.x / p.m_blocks);
    const int stride = (int)(gridDim.x / p.m_blocks), tiles = (p.N + 15) / 16;
    Codes<X, NB> c[DEPTH];   // (the last one's loads are on their way while the first is worked on)
    if constexpr (DEPTH == 2)
        if (first < tiles) c[0].load(p, first, wave, l, q);
    Fragment<X> x[NB][MT];
    const auto hold = [&](auto ends) {
        constexpr Ends ENDS = decltype(ends)::value;
        typedef typename X::T T;
        if constexpr (X::kStaged) {
            // A lane's vectors of a row lie far apart, and a load of them would touch 64
            // cache lines; so rows are loaded as they lie, and change places in LDS.
            constexpr int NE = 16 / sizeof(T), C = 128 * G / NE, V = Fragment<X>::kVectors;
            u32x4* own = stage[wave];
#pragma unroll
            for (int b = 0; b < NB / G; ++b)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < G * V; ++i) {
                        const int at = i * 64 + lane, m = min(m0 + 16 * t + at / C, p.M - 1);
                        const int k = (b * kWaves + wave) * 128 * G + at % C * NE;
                        x[b * G + i / V][t].put(i % V, load16<ENDS>((const T*)p.x + m * p.sx, k, p.K));
                    }
#pragma unroll
            for (int b = 0; b < NB / G; ++b)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
#pragma unroll
                    for (int i = 0; i < G * V; ++i) {
                        const int at = i * 64 + lane;
                        own[at / C * (C + 1) + at % C] = x[b * G + i / V][t].get(i % V);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int i = 0; i < G * V; ++i)
                        x[b * G + i / V][t].put(i % V, own[l * (C + 1) + Fragment<X>::at(i % V, q, i / V, G) / NE]);
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
        } else {
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int m = min(m0 + 16 * t + l, p.M - 1);
                    const auto of = [&](int quarter) { return ((j / G * kWaves + wave) * 4 + quarter) * G + j % G; };
                    x[j][t].template load<ENDS>((const T*)p.x + m * p.sx, of, q, p.K);
                }
        }
    };
    if (p.K % (16 / (int)sizeof(typename X::T)) == 0) hold(std::integral_constant<Ends, kEven>());
    else hold(std::integral_constant<Ends, kAny>());
    // A tile's sums of this wave.  The waves meet every TURNS tiles only, so that one may be
    // ahead of another (16 x 8192 to 114688, bf16: 141 us with one, 128 with two, 121 with
    // four).
    const auto work = [&](const Codes<X, NB>& c, int turn, int buf) {
        f32x4 acc[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if constexpr (kHidden<X, MT, NB>)
#pragma unroll
                for (int t = 0; t < MT; ++t) x[j][t].hide();
            multiply(c.codes[j], c.power[j / G] >> 8 * (j % G) & 255, x[j], acc);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) join[buf][turn][wave][t][lane] = acc[t];
    };
    for (int tile = first, buf = 0; tile < tiles; tile += TURNS * stride, buf ^= 1) {
        int turns = 0;
#pragma unroll
        for (int h = 0; h < TURNS; ++h) {
            const int now = tile + h * stride, then = now + (DEPTH - 1) * stride;
            if (now >= tiles) break;
            if (then < tiles) c[(h + DEPTH - 1) % DEPTH].load(p, then, wave, l, q);
            work(c[h % DEPTH], h, buf);
            ++turns;
        }
        __syncthreads();   // (the other buffer is read by no wave that is not past the last one)
        for (int e = threadIdx.x; e < turns * 256 * MT; e += kWaves * 64) {
            const int turn = e / (256 * MT), in = e % (256 * MT);
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum += ((const float*)join[buf][turn][w])[in];
            const int at = in % 256 / 4, row = m0 + in / 256 * 16 + at % 16;
            const int col = (tile + turn * stride) * 16 + at / 16 * 4 + in % 4;
            if (row < p.M && col < p.N) put((Y*)p.y + row * p.sy + col, p.scale ? sum * p.scale[row] : sum);
        }
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

constexpr int kGroups = 2;   // of 32 k that a lane of the split kernel takes at once

template <class X, class Y, int R, int MT, int WK>
hipError_t go(Fp4Params p, hipStream_t st) {
    constexpr int rows = 16 * R * (kWaves / WK), ahead = MT == 1 ? 2 : 1;
    p.m_blocks = (p.M + 16 * MT - 1) / (16 * MT);
    const int64_t blocks = (int64_t)((p.N + rows - 1) / rows) * p.m_blocks;   // (at most kMostTiles)
    hipLaunchKernelGGL((swr_fp4_kernel<X, Y, R, MT, kGroups, WK, ahead>), dim3((unsigned)blocks), dim3(kWaves * 64), 0,
                       st, p);
    return hipGetLastError();
}

// The split kernel's waves along k: as many as there are blocks of k for them.
// (Fewer waves along k and more along the rows were slower or the same at every size
// tried: one row of 4096 against 4096, 5.0 us with 8 along k, 7.3 with 4, 11.6 with 2;
// of 8192 against 28672, 45, 44 and 47.)
template <class X, class Y, int R, int MT>
hipError_t split(const Fp4Params& p, hipStream_t st) {
    const int blocks = (p.K + 128 * kGroups - 1) / (128 * kGroups);
    if (blocks == 1) return go<X, Y, R, MT, 1>(p, st);
    if (blocks <= 3) return go<X, Y, R, MT, 2>(p, st);
    if (blocks <= 7) return go<X, Y, R, MT, 4>(p, st);
    return go<X, Y, R, MT, 8>(p, st);
}

template <class X, class Y, int MT, int NB>
hipError_t hold(Fp4Params p, hipStream_t st) {
    if constexpr (held<X, MT, NB>() > kMostHeld) return hipErrorInvalidValue;   // (fits() is false)
    else {
        p.m_blocks = (p.M + 16 * MT - 1) / (16 * MT);
        const int64_t tiles = (p.N + 15) / 16, most = std::max(kCus / p.m_blocks, 1);
        // A second tile's codes on their way, where the registers have room for them
        // (a third's lost 1 % at 16 x 8192 bf16 rows against 28672).
        constexpr int depth = held<X, MT, NB>() + 2 * 5 * NB + (kHidden<X, MT, NB> ? 32 : 0) <= 224 ? 2 : 1;
        hipLaunchKernelGGL((swr_fp4_held_kernel<X, Y, MT, NB, depth>),
                           dim3((unsigned)(std::min(tiles, most) * p.m_blocks)), dim3(kWaves * 64), 0, st, p);
        return hipGetLastError();
    }
}

// Blocks of 128 k of a wave, as the held kernel is built for them; 0 past its last.
int blocks_a_wave(int K) {
    const int nb = ((K + 127) / 128 + kWaves - 1) / kWaves;
    return nb <= 2 ? nb : nb <= 4 ? 4 : nb <= 6 ? 6 : nb <= 8 ? 8 : 0;
}

template <class X, int MT>
bool fits(int K) {
    const int nb = blocks_a_wave(K);
    return nb != 0 && held<X, MT, 1>() * nb <= kMostHeld;
}

template <class X, class Y, int MT>
hipError_t hold(const Fp4Params& p, hipStream_t st) {
    switch (blocks_a_wave(p.K)) {
        case 1: return hold<X, Y, MT, 1>(p, st);
        case 2: return hold<X, Y, MT, 2>(p, st);
        case 4: return hold<X, Y, MT, 4>(p, st);
        case 6: return hold<X, Y, MT, 6>(p, st);
        default: return hold<X, Y, MT, 8>(p, st);
    }
}

// Which kernel, in us (split with one tile of W a wave, with two, held):
//     rows of x     2048 to 6176      4096 to 4096      8192 to 4096      8192 to 8192      8192 to 28672
//     1 bf16        4.6  4.4  4.7     4.6  6.6  6.1     8.1 11.6 10.6    12.4 13.3 14.1     45  39  35
//     8 bf16        5.9  5.0  4.7     6.2  7.7  6.3    10.1 13.3 10.9    17.7 14.8 14.3     71  60  35
//     8 8-bit       4.9  4.5  4.6     5.2  6.7  5.4     8.7 11.2  9.2    13.7 13.3 13.2     44  44  33
//     16 bf16       7.4  5.8  4.8     8.8  9.3  6.4    15.2 17.2 11.3    27.0 19.0 14.2    107  84  35
//     1 float32     9.4  6.7  6.8     8.8 11.4   -     17.2 21.9   -     31.7 23.9   -     112  93   -
// The split kernel's lanes load x with a cache line for each of its rows, time after time; the
// held one's load it once, but before all else, which few rows and few tiles pay back only
// where x is short, of two blocks of 128 k a wave at most.  It has one block a CU (two: 10 %
// slower).  Past 16 rows of x it takes 32 at a time if they fit (64 x 4096 to 4096,
// bf16: 11.0 us, the split kernel 13.5).
// Two tiles a wave, past 256 of them, serve rows of float32 and several of bf16; they cost one row
// of 8192 to 8192 7 %, and 8-bit rows that do not fit more: 16384 to 8192, 18.4 us for one row with
// one tile, 24.9 with two (16 rows: 28.6 and 28.2).
template <class X, class Y>
hipError_t by_size(const Fp4Params& p, hipStream_t st) {
    const int tiles = (p.N + 15) / 16;
    if (p.M > 8 || tiles > 2 * kCus || p.K <= 2 * 128 * kWaves) {
        if (p.M > 16 && fits<X, 2>(p.K)) return hold<X, Y, 2>(p, st);
        if (fits<X, 1>(p.K)) return hold<X, Y, 1>(p, st);
    }
    if (p.M > 16) return split<X, Y, 2, 2>(p, st);
    return tiles <= kCus ? split<X, Y, 1, 1>(p, st) : split<X, Y, 2, 1>(p, st);
}

constexpr int64_t kMostTiles = (1 << 23) - 1;   // of y, 16 x 16, a block of 512 threads each at most: below 2^32 threads

}  // namespace

hipError_t launch_fp4(int dtype, int out_dtype, const Fp4Params& p, void* stream) {
    const int64_t m = ((int64_t)p.M + 15) / 16, n = ((int64_t)p.N + 15) / 16;
    if (m * n > kMostTiles) {   // y in two halves
        Fp4Params a = p, b = p;
        const int64_t half = (std::max(m, n) + 1) / 2 * 16, es = out_dtype == SWR_DTYPE_F32 ? 4 : 2;
        if (m >= n) {
            a.M = (int32_t)half;
            b.M -= a.M;
            b.x = (const char*)p.x + half * p.sx * (dtype == SWR_DTYPE_F32 ? 4 : dtype == SWR_DTYPE_BF16 ? 2 : 1);
            if (p.scale) b.scale += half;
            b.y = (char*)p.y + half * p.sy * es;
        } else {
            a.N = (int32_t)half;
            b.N -= a.N;
            b.codes += half * p.sc;
            b.powers += half * p.sp;
            b.y = (char*)p.y + half * es;
        }
        const hipError_t e = launch_fp4(dtype, out_dtype, a, stream);
        return e != hipSuccess ? e : launch_fp4(dtype, out_dtype, b, stream);
    }
    const hipStream_t st = (hipStream_t)stream;
    const bool f32 = out_dtype == SWR_DTYPE_F32;
    if (dtype == SWR_DTYPE_FP8) return f32 ? by_size<XFp8, float>(p, st) : by_size<XFp8, uint16_t>(p, st);
    if (dtype == SWR_DTYPE_BF16) return f32 ? by_size<XBf16, float>(p, st) : by_size<XBf16, uint16_t>(p, st);
    return f32 ? by_size<XF32, float>(p, st) : by_size<XF32, uint16_t>(p, st);
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
