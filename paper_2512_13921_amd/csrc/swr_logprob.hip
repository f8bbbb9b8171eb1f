// swr_logprob.hip -- log probabilities of given tokens, their rows' entropy and best
// alternatives, and the logits' gradient, on gfx950.
//
// A row is read once.  A thread keeps the largest logit m that it has met, and with
// d = (x - m) scale log2 e of its logits the sums s = sum 2^d and u = sum 2^d d; both are
// taken to a new m by a factor, and two threads' sums to a common one.  Then
//
//     lse = scale m + ln 2 log2 s,   logp = ln 2 (d[token] - log2 s),   entropy = ln 2 (log2 s - u / s)
//
// (m is subtracted first: of logits that are all a type's lowest value, as a mask leaves them, the
// products would overflow, and of large ones lose what differs.)
//
// Alternatives: a wave keeps the largest (logit, token) that it has met in its lanes, the largest
// first, and looks at a tile of logits one by one only where some lane's largest
// reaches the last of them.  The first tile's lanes' largest, sorted, give a bound to begin with.
//
// The gradient reads the logits again:
//     dlogits = scale p (dlse - dlogp - dentropy (log p + entropy)) + scale dlogp at the token
//
// What bounds it is the bytes, with the vector unit close behind: a logit takes 10 operations, of
// which the exponential counts four.
#include <algorithm>
#include <cfloat>

#include "swr_lm_launch.h"
#include "swr_vectors.h"

namespace swr {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kTileVectors = 4;   // 16-byte vectors of a thread's tile
constexpr int64_t kMostBlocks = 1 << 20;

struct Sums {
    float m, s, u;
};
// What d is taken from: m, or any number where no logit is above -infinity.
__device__ inline float origin(float m) { return m == -__builtin_inff() ? 0.0f : m; }
__device__ inline void raise(Sums& a, float m, float k) {   // to a larger m
    if (m == a.m || a.s == 0.0f) {   // (nothing so far: no sums to take along)
        a.m = m;
        return;
    }
    const float d = (a.m - m) * k, f = __builtin_amdgcn_exp2f(d);
    a.u = f > 0.0f ? f * fmaf(a.s, d, a.u) : 0.0f * a.s;   // (keeps NaN)
    a.s *= f;
    a.m = m;
}
__device__ inline Sums join(Sums a, Sums b, float k) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m, k);
    raise(b, m, k);
    return {m, a.s + b.s, a.u + b.u};
}

// A logit's and its token's place in the order of alternatives: a larger key is better.  NaN is above
// all numbers, zeros are equal, and of equal logits the lower token is better.
__device__ inline uint32_t ordered(float x) {
    x += 0.0f;
    if (x != x) return 0xffffffffu;
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float unordered(uint32_t k) {
    return as_float(k == 0xffffffffu ? 0x7fc00000u : k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ inline uint64_t key_of(float x, uint32_t token) { return (uint64_t)ordered(x) << 32 | (uint32_t)~token; }

__device__ inline uint64_t lane_of(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// A wave's best, the largest key in lane 0.
struct Best {
    uint64_t key = 0, last = 0;   // last: of lane top - 1; less than every key while there are fewer
    __device__ void insert(uint64_t k, int top) {
        const int at = __popcll(__ballot(key > k)), lane = threadIdx.x % 64;
        const uint64_t up = __shfl_up(key, 1);
        key = lane < at ? key : lane == at ? k : up;
        last = lane_of(key, top - 1);
    }
};

// The value of order `top` among a wave's 64, the largest first.
__device__ inline uint32_t order_statistic(uint32_t v, int top) {
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int size = 2; size <= 64; size *= 2)
#pragma unroll
        for (int reach = size / 2; reach > 0; reach /= 2) {
            const uint32_t other = (uint32_t)__shfl_xor((int)v, reach);
            const bool down = (lane & size) == 0, low = (lane & reach) == 0;
            v = down == low ? max(v, other) : min(v, other);
        }
    return (uint32_t)__builtin_amdgcn_readlane((int)v, top - 1);
}

// What a block leaves of its part of a row: sums, and its best keys.
struct Part {
    Sums sums;
    uint32_t none;   // (the keys behind them are 8-byte aligned)
};
__device__ inline Part* part_of(void* work, int64_t row, int parts, int part) {
    return (Part*)work + row * parts + part;
}
__device__ inline uint64_t* keys_of(void* work, int64_t rows, int64_t row, int parts, int part, int top) {
    return (uint64_t*)((Part*)work + rows * parts) + (row * parts + part) * top;
}

// A row's distribution: log p = (x - m) scale - ln 2 log2 s.
struct Row {
    float m, scale, bits;
    bool empty;   // no logit above -infinity
    __device__ Row(const Sums& a, float scale) : m(a.m), scale(scale), bits(log2f(a.s)), empty(a.s == 0.0f) {}
    __device__ float log(float x) const { return empty ? -__builtin_inff() : fmaf(x - m, scale, -kLn2 * bits); }
};
__device__ inline void finish(const LogProbParams& p, int64_t row, const Sums& a, float x, bool scored) {
    const Row r(a, p.scale);
    p.lse[row] = r.empty ? -__builtin_inff() : fmaf(a.m, p.scale, kLn2 * r.bits);
    p.logp[row] = scored ? r.log(x) : 0.0f;
    p.entropy[row] = r.empty ? 0.0f : kLn2 * (r.bits - a.u / a.s);
}

__device__ inline int64_t token_of(const LogProbParams& p, int64_t row) {
    return p.wide_tokens ? ((const int64_t*)p.tokens)[row] : ((const int32_t*)p.tokens)[row];
}

// Writes the `top` largest of n keys in LDS, each to its place: as many as are larger.
__device__ inline void write_best(const LogProbParams& p, int64_t row, const uint64_t* keys, int n, int thread, int threads,
                                  const Row& r) {
    for (int i = thread; i < n; i += threads) {
        const uint64_t own = keys[i];
        if (own == 0) continue;   // (a place that no logit took)
        int at = 0;
        for (int k = 0; k < n; ++k) at += keys[k] > own;
        if (at >= p.top) continue;
        p.top_logp[row * p.top + at] = r.log(unordered((uint32_t)(own >> 32)));
        p.top_tokens[row * p.top + at] = (int64_t)(uint32_t)~(uint32_t)own;
    }
}

// A row, or a part of it, by WAVES waves: one (four rows a block), or a block's.
template <class E, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void swr_logprob_kernel(LogProbParams p) {
    typedef typename E::store T;
    constexpr int NE = E::NE, kVectors = kTileVectors, kTile = NE * kVectors;
    constexpr int kLists = WAVES == 1 ? 4 : WAVES;
    __shared__ Sums sums[kLists];
    __shared__ uint64_t best_keys[TOP ? kLists * SWR_TOP_MOST : 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int t = WAVES == 1 ? lane : threadIdx.x, size = 64 * WAVES;
    const float k = p.scale * kLog2e;
    const int64_t items = p.rows * p.parts, step = WAVES == 1 ? gridDim.x * 4 : gridDim.x;
    // (Waves of a block with rows of their own go as often round as each other: barriers.)
    for (int64_t base = WAVES == 1 ? blockIdx.x * 4 : blockIdx.x; base < items; base += step) {
        const int64_t item = WAVES == 1 ? base + wave : base;
        const bool there = item < items;
        const int64_t row = there ? item / p.parts : 0;
        const int part = there ? (int)(item - row * p.parts) : 0;
        const T* x = (const T*)p.logits + row * p.sl;
        const int64_t tiles = (p.vocab + (int64_t)kTile * size - 1) / ((int64_t)kTile * size);
        const int64_t first = there ? tiles * part / p.parts : 0, last = there ? tiles * (part + 1) / p.parts : 0;
        Sums a{-__builtin_inff(), 0.0f, 0.0f};
        Best best;
        for (int64_t tile = first; tile < last; ++tile) {
            Slice<E, NE> v[kVectors];
            const int64_t at = tile * kTile * size + (int64_t)t * NE;
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                const int64_t e = at + (int64_t)i * size * NE;
                if (e + NE <= p.vocab) v[i].v[0] = ((const Loose<T>*)(x + e))->v;
                else {
                    T tail[NE];
#pragma unroll
                    for (int c = 0; c < NE; ++c) tail[c] = e + c < p.vocab ? x[e + c] : E::to(-__builtin_inff());
                    __builtin_memcpy(v[i].v, tail, sizeof v[i].v);
                }
            }
            float top = v[0][0];
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
#pragma unroll
                for (int c = 0; c < NE; ++c) top = fmaxf(top, v[i][c]);
            if (top > a.m) raise(a, top, k);
            const float m = origin(a.m);
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
#pragma unroll
                for (int c = 0; c < NE; ++c) {
                    const float d = (v[i][c] - m) * k, e = __builtin_amdgcn_exp2f(d);
                    a.s += e;
                    a.u = fmaf(e, fmaxf(d, -160.0f), a.u);   // (2^-160 is 0 in float32)
                }
            if constexpr (TOP) {
                bool odd = false;   // NaN, which a maximum passes over
#pragma unroll
                for (int i = 0; i < kVectors; ++i)
#pragma unroll
                    for (int c = 0; c < NE; ++c) odd |= v[i][c] != v[i][c];
                const uint32_t largest = odd ? 0xffffffffu : ordered(top);
                uint32_t bound = (uint32_t)(best.last >> 32);
                if (best.last == 0) bound = max(bound, order_statistic(at < p.vocab ? largest : 0, p.top));
                if (__ballot(largest >= bound && at < p.vocab)) {
#pragma unroll
                    for (int i = 0; i < kVectors; ++i)
#pragma unroll
                        for (int c = 0; c < NE; ++c) {
                            const int64_t token = at + (int64_t)i * size * NE + c;
                            const uint64_t own = key_of(v[i][c], (uint32_t)token);
                            const bool may = token < p.vocab && (uint32_t)(own >> 32) >= bound;
                            uint64_t left = __ballot(may && own > best.last);
                            while (left) {
                                const uint64_t cand = lane_of(own, __builtin_ctzll(left));
                                left &= left - 1;
                                if (cand > best.last) best.insert(cand, p.top);
                            }
                        }
                }
            }
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) {
            const Sums b{__shfl_xor(a.m, m), __shfl_xor(a.s, m), __shfl_xor(a.u, m)};
            // (both lanes add in the same order)
            a = lane & m ? join(b, a, k) : join(a, b, k);
        }
        uint64_t* own_keys = best_keys + (WAVES == 1 ? wave * SWR_TOP_MOST : 0);
        if constexpr (TOP) {
            if (lane < p.top) best_keys[WAVES == 1 ? wave * SWR_TOP_MOST + lane : wave * p.top + lane] = best.key;
        }
        if constexpr (WAVES > 1) {
            if (lane == 0) sums[wave] = a;
            __syncthreads();
            a = sums[0];
            for (int w = 1; w < WAVES; ++w) a = join(a, sums[w], k);
        } else if constexpr (TOP) {
            __syncthreads();
        }
        const int keys = TOP ? (WAVES == 1 ? 1 : WAVES) * p.top : 0;
        if (there && p.parts == 1) {
            const int64_t token = token_of(p, row);
            const bool scored = token >= 0 && token < p.vocab;
            if (t == 0) finish(p, row, a, scored ? E::one(x[token]) : 0.0f, scored);
            if constexpr (TOP) {
                write_best(p, row, own_keys, keys, t, size, Row(a, p.scale));
            }
        } else if (there) {
            if (t == 0) *part_of(p.work, row, p.parts, part) = Part{a, 0};
            if constexpr (TOP) {
                // The part's best, in any order; places that no key takes are 0.
                uint64_t* out = keys_of(p.work, p.rows, row, p.parts, part, p.top);
                for (int i = t; i < keys; i += size) {
                    const uint64_t own = own_keys[i];
                    int at = 0;
                    for (int q = 0; q < keys; ++q) at += own_keys[q] > own || (own_keys[q] == own && q < i);
                    if (at < p.top) out[at] = own;
                }
            }
        }
        if constexpr (WAVES > 1 || TOP) __syncthreads();   // (the LDS has been read)
    }
}

// Rows of several parts: their sums in order, and the best of their best.
template <class E, bool TOP>
__global__ __launch_bounds__(256) void swr_logprob_join_kernel(LogProbParams p) {
    __shared__ uint64_t list[SWR_TOP_MOST], next[2 * SWR_TOP_MOST];
    const float k = p.scale * kLog2e;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        Sums a = part_of(p.work, row, p.parts, 0)->sums;
        for (int i = 1; i < p.parts; ++i) a = join(a, part_of(p.work, row, p.parts, i)->sums, k);
        const int64_t token = token_of(p, row);
        const bool scored = token >= 0 && token < p.vocab;
        if (threadIdx.x == 0)
            finish(p, row, a, scored ? E::one(((const typename E::store*)p.logits)[row * p.sl + token]) : 0.0f, scored);
        if constexpr (TOP) {
            const int t = threadIdx.x;
            if (t < p.top) list[t] = keys_of(p.work, p.rows, row, p.parts, 0, p.top)[t];
            for (int part = 1; part < p.parts; ++part) {
                __syncthreads();
                if (t < p.top) next[t] = list[t];
                else if (t < 2 * p.top) next[t] = keys_of(p.work, p.rows, row, p.parts, part, p.top)[t - p.top];
                __syncthreads();
                if (t < 2 * p.top) {
                    const uint64_t own = next[t];
                    int at = 0;
                    for (int q = 0; q < 2 * p.top; ++q) at += next[q] > own || (next[q] == own && q < t);
                    if (at < p.top) list[at] = own;
                }
            }
            __syncthreads();
            write_best(p, row, list, p.top, t, 256, Row(a, p.scale));
            __syncthreads();
        }
    }
}

// The gradient: blockIdx.y's rows in turn, a thread's vectors 256 apart.
template <class E>
__global__ __launch_bounds__(256) void swr_logprob_back_kernel(LogProbParams p) {
    typedef typename E::store T;
    constexpr int NE = E::NE, kVectors = 2;
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const int64_t token = token_of(p, row);
        const bool scored = token >= 0 && token < p.vocab;
        const float lse = p.lse_in[row], entropy = p.entropy_in[row];
        const float dlogp = scored && p.dlogp ? p.dlogp[row] : 0.0f, dlse = p.dlse ? p.dlse[row] : 0.0f;
        const float dentropy = p.dentropy ? p.dentropy[row] : 0.0f;
        const bool empty = lse == -__builtin_inff();
        const float base = p.scale * (dlse - dlogp - dentropy * entropy), slope = -p.scale * dentropy;
        const float hit = p.scale * dlogp;
        const T* x = (const T*)p.logits + row * p.sl;
        T* out = (T*)p.dlogits + row * p.sd;
        for (int64_t at = ((int64_t)blockIdx.x * 256 * kVectors + threadIdx.x) * NE; at < p.vocab;
             at += (int64_t)gridDim.x * 256 * kVectors * NE) {
            Slice<E, NE> v[kVectors];
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                v[i] = {};
                if (at + (int64_t)i * 256 * NE < p.vocab) v[i].load(x, (int)(at + (int64_t)i * 256 * NE), (int)p.vocab);
            }
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                const int64_t e = at + (int64_t)i * 256 * NE;
                float f[NE];
#pragma unroll
                for (int c = 0; c < NE; ++c) {
                    const float logs = fmaf(v[i][c], p.scale, -lse);
                    const float prob = __builtin_amdgcn_exp2f(logs * kLog2e);
                    f[c] = prob * fmaf(slope, fmaxf(logs, -110.0f), base);   // (exp(-110) is 0 in float32)
                    if (empty) f[c] = 0.0f;
                    else if (e + c == token && scored) f[c] += hit;
                }
                if (e < p.vocab) store<E, NE>(out + e, (int)min(p.vocab - e, (int64_t)NE), f);
            }
        }
    }
}

unsigned grid_of(int64_t blocks) { return (unsigned)std::max<int64_t>(1, std::min(blocks, kMostBlocks)); }

// Waves of a row (or part).
int waves_of(int64_t vocab) { return vocab <= 2048 ? 1 : vocab <= 16384 ? 4 : 16; }

template <class E, bool TOP>
hipError_t forward(const LogProbParams& p, hipStream_t st) {
    const int waves = waves_of(p.vocab);
    const int64_t items = p.rows * p.parts;
    if (waves == 1)
        hipLaunchKernelGGL((swr_logprob_kernel<E, 1, TOP>), dim3(grid_of((items + 3) / 4)), dim3(256), 0, st, p);
    else if (waves == 4)
        hipLaunchKernelGGL((swr_logprob_kernel<E, 4, TOP>), dim3(grid_of(items)), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((swr_logprob_kernel<E, 16, TOP>), dim3(grid_of(items)), dim3(1024), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL((swr_logprob_join_kernel<E, TOP>), dim3(grid_of(p.rows)), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <class E>
hipError_t backward(const LogProbParams& p, hipStream_t st) {
    const int64_t blocks = std::min<int64_t>((p.vocab + 512 * E::NE - 1) / (512 * E::NE), 1 << 15);
    hipLaunchKernelGGL((swr_logprob_back_kernel<E>), dim3((unsigned)blocks, (unsigned)std::min<int64_t>(p.rows, 32768)),
                       dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace

// Blocks that share a row: where few rows leave the GPU idle.
int logprob_parts(int64_t rows, int64_t vocab) {
    if (waves_of(vocab) < 16) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(vocab / 65536, 256 / std::max<int64_t>(rows, 1)));
}

int64_t logprob_work_bytes(int64_t rows, int64_t vocab, int top) {
    const int parts = logprob_parts(rows, vocab);
    return parts > 1 ? rows * parts * ((int64_t)sizeof(Part) + 8 * top) : 0;
}

hipError_t launch_logprob(int dtype, const LogProbParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == SWR_DTYPE_F32) return p.top ? forward<F32, true>(p, st) : forward<F32, false>(p, st);
    return p.top ? forward<Bf16, true>(p, st) : forward<Bf16, false>(p, st);
}

hipError_t launch_logprob_backward(int dtype, const LogProbParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    return dtype == SWR_DTYPE_F32 ? backward<F32>(p, st) : backward<Bf16>(p, st);
}

}  // namespace swr
