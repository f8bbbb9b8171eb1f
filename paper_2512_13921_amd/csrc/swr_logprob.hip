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
// Alternatives: of the threads' largest logits the one of order `top` is a bound that as many logits reach, and few
// more: the few threads that have some look through theirs once more and put them into a list, which is
// then ranked.  (With sorted lists that took in logits as they were met, 8 rows of 65536 took 40 us.)
//
// The gradient reads the logits again:
//     dlogits = scale p (dlse - dlogp - dentropy (log p + entropy)) + scale dlogp at the token
//
// What bounds it is the bytes, with the vector unit close behind: a logit takes 10 operations, of
// which the exponential counts two.  4095 rows of 65536 bf16 take 100 us forward (5.4 TB/s) and 195 for the gradient (5.5);
// 8 rows with 20 alternatives 18, in launches and what each waits for.
#include <algorithm>
#include <cfloat>
#include <type_traits>

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

// ... of a wave's lanes; every lane adds in the same order.
__device__ inline Sums wave_join(Sums a, float k) {
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
        const Sums b{__shfl_xor(a.m, m), __shfl_xor(a.s, m), __shfl_xor(a.u, m)};
        a = lane & m ? join(b, a, k) : join(a, b, k);
    }
    return a;
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
__device__ inline uint32_t partner(uint32_t v, int reach) { return (uint32_t)__shfl_xor((int)v, reach); }
__device__ inline uint64_t partner(uint64_t v, int reach) { return (uint64_t)__shfl_xor((long long)v, reach); }

// A wave's 64 values in its lanes, the largest first.
__device__ inline uint32_t sorted(uint32_t v) {
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int size = 2; size <= 64; size *= 2)
#pragma unroll
        for (int reach = size / 2; reach > 0; reach /= 2) {
            const uint32_t other = partner(v, reach);
            const bool down = (lane & size) == 0, low = (lane & reach) == 0;
            v = down == low ? max(v, other) : min(v, other);
        }
    return v;
}
// The 64 largest of two such lists, of the second in reverse (its last value in lane 0).
template <class T>
__device__ inline T merged(T v, T reverse) {
    const int lane = threadIdx.x % 64;
    v = max(v, reverse);
#pragma unroll
    for (int reach = 32; reach > 0; reach /= 2) {
        const T other = partner(v, reach);
        v = lane & reach ? min(v, other) : max(v, other);
    }
    return v;
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

// How many of n keys are larger.
__device__ inline int rank_of(const uint64_t* keys, int n, uint64_t own) {
    int at = 0;
#pragma unroll 8
    for (int k = 0; k < n; ++k) at += keys[k] > own;
    return at;
}
__device__ inline void write_one(const LogProbParams& p, int64_t row, int at, uint64_t key, const Row& r) {
    p.top_logp[row * p.top + at] = r.log(unordered((uint32_t)(key >> 32)));
    p.top_tokens[row * p.top + at] = (int64_t)(uint32_t)~(uint32_t)key;
}

// The lists that a row's alternatives are found with: logits above the bound, and equal to it.
constexpr int kAbove = 1024, kEqual = 256;
template <int WAVES>
struct Lists {
    uint64_t above[WAVES == 1 ? 512 : kAbove], equal[kEqual];
    uint32_t largest[WAVES == 1 ? 1 : WAVES][64];   // the waves' lists
    int counts[WAVES];
    int above_n, equal_n;
    uint32_t bound;
    static constexpr int kMost = WAVES == 1 ? 512 : kAbove;
};

// The threads of a row wait for each other.
template <int WAVES>
__device__ inline void meet() {
    if constexpr (WAVES == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup"), __builtin_amdgcn_wave_barrier();
    else __syncthreads();
}

// The `top` largest keys of the elements first .. last - 1 of a row, in any order of the row's threads: f(rank, key)
// for each, where there are as many.  `own`: the largest of the thread's own, 0 without any.
template <class E, int WAVES, class F>
__device__ inline void find_best(const typename E::store* x, int64_t first, int64_t last, int top, uint32_t own, int t,
                                 Lists<WAVES>& l, F f) {
    constexpr int NE = E::NE, kThreads = 64 * WAVES;
    const int lane = threadIdx.x % 64, wave = t / 64;
    uint32_t in_order = sorted(own);
    for (int step = WAVES / 2; step > 0; step /= 2) {
        if (wave < 2 * step) l.largest[wave][lane] = in_order;
        __syncthreads();
        if (wave < step) in_order = merged(in_order, l.largest[wave + step][63 - lane]);
        __syncthreads();
    }
    if (t == top - 1) l.bound = in_order;
    for (;;) {
        if (t == 0) l.above_n = l.equal_n = 0;
        meet<WAVES>();
        const uint32_t bound = l.bound;
        // A wave looks through the elements of those of its lanes that have some, one lane's after the other's:
        // short code, as it runs once (unrolled, it took 5 us more, to be fetched).
        for (uint64_t todo = __ballot(own >= bound && own > 0); todo; todo &= todo - 1) {
            const int64_t who = first + ((int64_t)wave * 64 + __builtin_ctzll(todo)) * NE;
#pragma unroll 1
            for (int64_t from = 0; who + from * kThreads < last; from += 64) {
                const int64_t e = who + (from + lane / NE * NE) * kThreads + lane % NE;
                const uint32_t v = e < last ? ordered(E::one(x[e])) : 0;
                const uint64_t key = (uint64_t)v << 32 | (uint32_t)~(uint32_t)e, before = ((uint64_t)1 << lane) - 1;
                const uint64_t more = __ballot(v > bound), same = __ballot(v == bound && e < last);
                int to = 0;
                if (lane == 0 && more) to = atomicAdd(&l.above_n, __popcll(more));
                to = __builtin_amdgcn_readfirstlane(to) + __popcll(more & before);
                if (v > bound && to < Lists<WAVES>::kMost) l.above[to] = key;
                if (lane == 0 && same) to = atomicAdd(&l.equal_n, __popcll(same));
                to = __builtin_amdgcn_readfirstlane(to) + __popcll(same & before);
                if (v == bound && e < last && to < kEqual) l.equal[to] = key;
            }
        }
        meet<WAVES>();
        const int above = l.above_n, equal = l.equal_n;
        if (above > Lists<WAVES>::kMost) {   // too many: the bound of order `top` among those that are listed
            for (int i = t; i < Lists<WAVES>::kMost; i += kThreads)
                if (rank_of(l.above, Lists<WAVES>::kMost, l.above[i]) == top - 1) l.bound = (uint32_t)(l.above[i] >> 32);
            meet<WAVES>();
            continue;
        }
        int ties = equal;
        if (equal > kEqual) {   // many equal ones: the first of them, in order
            const int need = max(top - above, 0);
            int so_far = 0;
            for (int64_t base = first; base < last && so_far < need; base += kThreads) {
                const int64_t e = base + t;
                const bool is = e < last && ordered(E::one(x[min(e, last - 1)])) == bound;
                const uint64_t mask = __ballot(is);
                int before = so_far, all = __popcll(mask);
                if constexpr (WAVES > 1) {
                    if (lane == 0) l.counts[wave] = all;
                    __syncthreads();
                    all = 0;
                    for (int w = 0; w < WAVES; ++w) {
                        before += w < wave ? l.counts[w] : 0;
                        all += l.counts[w];
                    }
                    __syncthreads();
                }
                before += __popcll(mask & (((uint64_t)1 << lane) - 1));
                if (is && before < need) l.equal[before] = (uint64_t)bound << 32 | (uint32_t)~(uint32_t)e;
                so_far += all;
            }
            ties = min(so_far, need);
            meet<WAVES>();
        }
        for (int i = t; i < above; i += kThreads) {
            const int at = rank_of(l.above, above, l.above[i]);
            if (at < top) f(at, l.above[i]);
        }
        for (int i = t; i < ties; i += kThreads) {
            const int at = above + rank_of(l.equal, ties, l.equal[i]);
            if (at < top) f(at, l.equal[i]);
        }
        meet<WAVES>();   // (the lists have been read)
        return;
    }
}

// A row, or a part of it, by WAVES waves: one (four rows a block), or a block's.
template <class E, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void swr_logprob_kernel(LogProbParams p) {
    typedef typename E::store T;
    constexpr int NE = E::NE, kVectors = kTileVectors, kTile = NE * kVectors;
    constexpr int kLists = WAVES == 1 ? 4 : WAVES;
    __shared__ Sums sums[kLists];
    struct None {};
    __shared__ std::conditional_t<TOP, Lists<WAVES>, None> lists[TOP && WAVES == 1 ? 4 : 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int t = WAVES == 1 ? lane : threadIdx.x, size = 64 * WAVES;
    const float k = p.scale * kLog2e;
    const int64_t items = p.rows * p.parts, step = WAVES == 1 ? gridDim.x * 4 : gridDim.x;
    for (int64_t base = WAVES == 1 ? blockIdx.x * 4 : blockIdx.x; base < items; base += step) {
        const int64_t item = WAVES == 1 ? base + wave : base;
        const bool there = item < items;
        const int64_t row = there ? item / p.parts : 0;
        const int part = there ? (int)(item - row * p.parts) : 0;
        const T* x = (const T*)p.logits + row * p.sl;
        const int64_t tiles = (p.vocab + (int64_t)kTile * size - 1) / ((int64_t)kTile * size);
        const int64_t first = there ? tiles * part / p.parts : 0, last = there ? tiles * (part + 1) / p.parts : 0;
        Sums a{-__builtin_inff(), 0.0f, 0.0f};
        bool odd = false;   // a NaN, which a maximum passes over
        struct Tile {
            u32x4 v[kVectors];
        } even, odd_tile;
        const auto fetch = [&](Tile& tile, int64_t at) {   // a whole tile
            const T* from = x + at * kTile * size + (int64_t)t * NE;
#pragma unroll
            for (int i = 0; i < kVectors; ++i) tile.v[i] = ((const Loose<T>*)(from + (int64_t)i * size * NE))->v;
        };
        const auto take = [&](const Tile& tile) {
            float top = E::get(tile.v[0], 0);
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
#pragma unroll
                for (int c = 0; c < NE; ++c) top = fmaxf(top, E::get(tile.v[i], c));
            if (top > a.m) raise(a, top, k);
            const float m = origin(a.m);
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
#pragma unroll
                for (int c = 0; c < NE; ++c) {
                    const float d = (E::get(tile.v[i], c) - m) * k, e = __builtin_amdgcn_exp2f(d);
                    a.s += e;
                    a.u = fmaf(e, fmaxf(d, -160.0f), a.u);   // (2^-160 is 0 in float32)
                }
            if constexpr (TOP) {
#pragma unroll
                for (int i = 0; i < kVectors; ++i)
#pragma unroll
                    for (int c = 0; c < NE; ++c) odd |= E::get(tile.v[i], c) != E::get(tile.v[i], c);
            }
        };
        // Whole tiles, the next one's loads ahead; then one that the row ends in.
        const int64_t whole = min(last, p.vocab / ((int64_t)kTile * size));
        if (first < whole) fetch(even, first);
        for (int64_t tile = first; tile < whole; tile += 2) {
            fetch(odd_tile, min(tile + 1, whole - 1));
            take(even);
            if (tile + 1 >= whole) break;
            fetch(even, min(tile + 2, whole - 1));
            take(odd_tile);
        }
        if (max(first, whole) < last) {
            const int64_t at = max(first, whole) * kTile * size + (int64_t)t * NE;
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                const int64_t e = at + (int64_t)i * size * NE;
                if (e + NE <= p.vocab) even.v[i] = ((const Loose<T>*)(x + e))->v;
                else {
                    T tail[NE];
#pragma unroll
                    for (int c = 0; c < NE; ++c) tail[c] = e + c < p.vocab ? x[e + c] : E::to(-__builtin_inff());
                    __builtin_memcpy(&even.v[i], tail, sizeof even.v[i]);
                }
            }
            take(even);
        }
        const int64_t begin = first * kTile * size, end = min(last * kTile * size, p.vocab);
        uint32_t largest = 0;
        if (TOP && begin + (int64_t)t * NE < end) largest = odd ? 0xffffffffu : ordered(a.m);
        a = wave_join(a, k);
        if constexpr (WAVES > 1) {
            if (lane == 0) sums[wave] = a;
            __syncthreads();
            a = sums[0];
            for (int w = 1; w < WAVES; ++w) a = join(a, sums[w], k);
        }
        if (there && p.parts == 1) {
            const int64_t token = token_of(p, row);
            const bool scored = token >= 0 && token < p.vocab;
            if (t == 0) finish(p, row, a, scored ? E::one(x[token]) : 0.0f, scored);
            if constexpr (TOP) {
                const Row r(a, p.scale);
                find_best<E, WAVES>(x, begin, end, p.top, largest, t, lists[WAVES == 1 ? wave : 0],
                                    [&](int at, uint64_t key) { write_one(p, row, at, key, r); });
            }
        } else if (there) {
            if (t == 0) *part_of(p.work, row, p.parts, part) = Part{a, 0};
            if constexpr (TOP) {
                uint64_t* out = keys_of(p.work, p.rows, row, p.parts, part, p.top);
                if (t < p.top) out[t] = 0;   // (a part may have fewer logits)
                find_best<E, WAVES>(x, begin, end, p.top, largest, t, lists[WAVES == 1 ? wave : 0],
                                    [&](int at, uint64_t key) { out[at] = key; });
            }
        }
        if constexpr (WAVES > 1) __syncthreads();   // (the LDS has been read)
    }
}

// Rows of several parts: their sums in order, and the best of their best, which four waves merge.
template <class E, bool TOP>
__global__ __launch_bounds__(256) void swr_logprob_join_kernel(LogProbParams p) {
    __shared__ uint64_t lists[4][64];
    const float k = p.scale * kLog2e;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const int64_t token = token_of(p, row);
        const bool scored = token >= 0 && token < p.vocab;
        const float x = scored ? E::one(((const typename E::store*)p.logits)[row * p.sl + token]) : 0.0f;
        Sums a{-__builtin_inff(), 0.0f, 0.0f};   // (of at most 64 parts, one a lane)
        if (lane < p.parts) a = part_of(p.work, row, p.parts, lane)->sums;
        a = wave_join(a, k);
        if (threadIdx.x == 0) finish(p, row, a, x, scored);
        if constexpr (TOP) {
            uint64_t best = 0;
            for (int part = wave; part < p.parts; part += 4) {
                const uint64_t* list = keys_of(p.work, p.rows, row, p.parts, part, p.top);
                best = merged(best, 63 - lane < p.top ? list[63 - lane] : 0);
            }
            lists[wave][lane] = best;
            __syncthreads();
            if (wave == 0) {
                for (int w = 1; w < 4; ++w) best = merged(best, lists[w][63 - lane]);
                if (lane < p.top) write_one(p, row, lane, best, Row(a, p.scale));
            }
            __syncthreads();
        }
    }
}

// The gradient: blockIdx.y's rows in turn, a thread's vectors 256 apart.
//
// lse as a float32 is off by half its last place, and p by as much of itself: 2^-17 up to 256.  Of a row farther out (all
// of a type's lowest value, say, where nothing of log V is left in lse, or which is infinite as a float32 though no logit
// is) one block takes the largest logit and the sum anew, finds whether there is a logit above -infinity at all, and writes the
// row's gradient: it has read the row before it writes to it, as a call in place needs.  4095 far rows of 65536 bf16 take 440 us,
// ordinary ones 195 (4757 with all of a row's blocks at it, each for itself).
constexpr float kFar = 256.0f;
// A row's largest logit and its sum by a block.  (A function of its own, and one vector of a thread at a time, for the
// registers: of 4095 rows of 65536 bf16 the kernel takes 195 us, 210 with four vectors, of 91 registers for 80; with these
// lines in the kernel it took 211.)
template <class E>
__device__ __attribute__((noinline)) Sums anew(const typename E::store* x, int64_t vocab, float k, Sums* sums) {
    constexpr int NE = E::NE;
    Sums a{-__builtin_inff(), 0.0f, 0.0f};
#pragma unroll 1
    for (int64_t e = (int64_t)threadIdx.x * NE; e < vocab; e += 256 * NE) {
        u32x4 v;
        if (e + NE <= vocab) v = ((const Loose<typename E::store>*)(x + e))->v;
        else {
            typename E::store tail[NE];
#pragma unroll
            for (int c = 0; c < NE; ++c) tail[c] = e + c < vocab ? x[e + c] : E::to(-__builtin_inff());
            __builtin_memcpy(&v, tail, sizeof v);
        }
        float top = E::get(v, 0);
#pragma unroll
        for (int c = 1; c < NE; ++c) top = fmaxf(top, E::get(v, c));
        if (top > a.m) raise(a, top, k);
        const float m = origin(a.m);
#pragma unroll
        for (int c = 0; c < NE; ++c) a.s += __builtin_amdgcn_exp2f((E::get(v, c) - m) * k);
    }
    a = wave_join(a, k);
    __syncthreads();   // (the last row's have been read)
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = a;
    __syncthreads();
    return join(join(sums[0], sums[1], k), join(sums[2], sums[3], k), k);
}
// A block's own value, in a scalar register.
__device__ inline float uniform(float v) {
    return as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__builtin_bit_cast(uint32_t, v)));
}
template <class E>
__global__ __launch_bounds__(256) void swr_logprob_back_kernel(LogProbParams p) {
    typedef typename E::store T;
    constexpr int NE = E::NE, kVectors = 2;
    __shared__ Sums sums[4];
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const int64_t token = token_of(p, row);
        const bool scored = token >= 0 && token < p.vocab;
        const float lse = p.lse_in[row], entropy = p.entropy_in[row];
        const float dlogp = scored && p.dlogp ? p.dlogp[row] : 0.0f, dlse = p.dlse ? p.dlse[row] : 0.0f;
        const float dentropy = p.dentropy ? p.dentropy[row] : 0.0f;
        float base = uniform(p.scale * (dlse - dlogp - dentropy * entropy)), slope = uniform(-p.scale * dentropy);
        float hit = uniform(p.scale * dlogp);
        const T* x = (const T*)p.logits + row * p.sl;
        T* out = (T*)p.dlogits + row * p.sd;
        // log p = (x - m) scale - off
        float m = 0.0f, off = lse;
        int64_t block = blockIdx.x, blocks = gridDim.x;   // of the row
        // Far rows (none with NaN).  Where p does not count it is taken as 0: by their lse, as far from the logits as that may
        // lie, it could be infinite, and its product with 0 no number.  (The token's own gradient needs to know of an empty row.)
        if (fabsf(lse) > kFar) {
            if (base == 0.0f && slope == 0.0f && (hit == 0.0f || fabsf(lse) < __builtin_inff())) {
                off = __builtin_inff();
            } else {
                // (rows' blocks go to the 8 dies in turn, and so do one of each)
                if (block != row % blocks) continue;
                block = 0;
                blocks = 1;
                const Sums a = anew<E>(x, p.vocab, p.scale * kLog2e, sums);
                const bool empty = uniform(a.s) == 0.0f;   // (no logit above -infinity: p, and every gradient, is 0)
                m = uniform(origin(a.m));
                off = uniform(empty ? __builtin_inff() : kLn2 * log2f(a.s));
                if (empty) base = slope = hit = 0.0f;
            }
        }
        for (int64_t at = (block * 256 * kVectors + threadIdx.x) * NE; at < p.vocab;
             at += blocks * 256 * kVectors * NE) {
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
                    const float logs = fmaf(v[i][c] - m, p.scale, -off);
                    const float prob = __builtin_amdgcn_exp2f(logs * kLog2e);
                    f[c] = prob * fmaf(slope, fmaxf(logs, -110.0f), base);   // (exp(-110) is 0 in float32)
                    if (e + c == token && scored) f[c] += hit;
                }
                if (e < p.vocab) store<E, NE>(out + e, (int)min(p.vocab - e, (int64_t)NE), f);
            }
        }
    }
}

unsigned grid_of(int64_t blocks) { return (unsigned)std::max<int64_t>(1, std::min(blocks, kMostBlocks)); }

// Waves of a row (or part), which take 32 (float32: 16) logits a lane at a time: 16 where there are too few rows (or
// parts) for the GPU's compute units to have more than two each.
int waves_of(int64_t rows, int64_t vocab, int parts) {
    return vocab <= 2048 ? 1 : vocab <= 16384 || parts > 1 || rows > 512 ? 4 : 16;
}

template <class E, bool TOP>
hipError_t forward(const LogProbParams& p, hipStream_t st) {
    const int waves = waves_of(p.rows, p.vocab, p.parts);
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

// Blocks that share a row: where few rows leave the GPU idle, about as many as there are compute units, and
// parts of 8192 logits and more.
int logprob_parts(int64_t rows, int64_t vocab) {
    if (vocab <= 16384 || rows > 64) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(vocab / 8192, 64),
                                                               256 / std::max<int64_t>(rows, 1)));
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
