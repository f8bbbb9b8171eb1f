// swr_scan.hip -- selective state space scan on gfx950: forward, backward and
// single tokens.
//
//     s = softplus(dt + bias);   a = exp(s A);   h = a h + (s x) B;
//     v = C . h + skip x;        y = v z sigma(z)
//
// and backwards, with w = dy z sigma(z) and G the gradient that reaches h_t from
// later tokens through a_(t+1):
//
//     g = C w + G;   dC = w h;   dB = g (s x);   G' = a g
//     ds = x (g . B) + (G' h_(t-1)) . A;   dA = sum s G' h_(t-1);   dx = s (g . B) + skip w
//
// A channel's states are shared out over L lanes of a wave, S states each, so that
// the sums over states stay within 16 lanes (DPP) and the states in registers
// over a whole run of tokens.  Tokens go in tiles of 16: what a token has to itself
// (its step, the gates) is worked out once, by one of its channel's L lanes, and
// handed to the others; B and C of a tile are in LDS as floats, read by all.
//
// What bounds it is not the bytes but the vector unit: of each state a token takes an
// exponential (a quarter of the rate), two products and two multiply-adds, 32
// cycles of a SIMD for a wave's 64 states.
//
// Where the channels alone do not fill the GPU, a sequence is cut into runs:
// the first pass finds each run's states from zero and the sum of its steps (the
// product of its decays is exp(A times that)), the second chains them, the third
// runs over the tokens with the right states.  The backward's runs go the same way
// from the end.
#include <algorithm>
#include <cfloat>
#include <utility>

#include "swr_lm_launch.h"
#include "swr_vectors.h"

namespace swr {
namespace {

constexpr int kTile = SWR_SCAN_BLOCK;
constexpr int kWaves = 4;
constexpr float kLog2e = 1.44269504088896340736f;

template <class F, int... I>
__device__ inline void each_of(std::integer_sequence<int, I...>, F&& f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ inline void each(F&& f) { each_of(std::make_integer_sequence<int, N>{}, f); }

template <int CTRL>
__device__ inline float dpp(float v) {
    return as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__builtin_bit_cast(uint32_t, v), CTRL, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140, kRotate4 = 0x124, kRotate8 = 0x128;

// v of lane J of every L lanes.
template <int L, int J>
__device__ inline float from_lane(float v) {
    if constexpr (L == 1) return v;
    else if constexpr (L == 2) return dpp<J | J << 2 | (2 + J) << 4 | (2 + J) << 6>(v);
    else if constexpr (L == 4) return dpp<J | J << 2 | J << 4 | J << 6>(v);
    else
        return as_float((uint32_t)__builtin_amdgcn_ds_swizzle((int)__builtin_bit_cast(uint32_t, v),
                                                              J << 5 | (31 & ~(L - 1))));
}
// Sum over every L lanes; all of them get it.
template <int L>
__device__ inline float lane_sum(float v) {
    if constexpr (L >= 2) v += dpp<kXor1>(v);
    if constexpr (L >= 4) v += dpp<kXor2>(v);
    if constexpr (L >= 8) v += dpp<kHalfMirror>(v);
    if constexpr (L >= 16) v += dpp<kMirror>(v);
    return v;
}

// log(1 + exp(v)) and its derivative.  With e = exp(-|v|) and r = e / (2 + e),
// log(1 + e) = 2 artanh(r) = 2 (r + r^3 / 3 + ...), r at most 1/3: the terms left out are
// under 2e-8 of it, and small steps (v far below 0) keep their relative precision.
struct Softplus {
    float value, slope;
    __device__ explicit Softplus(float v) {
        const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v));
        const float r = e * __builtin_amdgcn_rcpf(2.0f + e), q = r * r;
        float s = 1.0f / 13.0f;
        s = fmaf(s, q, 1.0f / 11.0f);
        s = fmaf(s, q, 1.0f / 9.0f);
        s = fmaf(s, q, 1.0f / 7.0f);
        s = fmaf(s, q, 1.0f / 5.0f);
        s = fmaf(s, q, 1.0f / 3.0f);
        s = fmaf(s, q, 1.0f);
        value = fmaf(2.0f * r, s, v > 0.0f ? v : 0.0f);
        const float half = __builtin_amdgcn_rcpf(1.0f + e);
        slope = v >= 0.0f ? half : e * half;
    }
};
__device__ inline float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v));
}

// A finite rate in place of an infinite one, so that a step of zero leaves the
// state as it is; exp of its product with any other step is the same.
__device__ inline float finite(float v) { return v < -FLT_MAX ? -FLT_MAX : v > FLT_MAX ? FLT_MAX : v; }

// S states of a channel from state n on; zeros past the N that there are.
template <int S, bool FULL>
__device__ inline void load_states(const float* p, int n, int N, float* h) {
    if constexpr (FULL) {
#pragma unroll
        for (int i = 0; i < S; i += 4) {
            const u32x4 v = ((const Loose<float>*)(p + n + i))->v;
#pragma unroll
            for (int k = 0; k < 4; ++k) h[i + k] = as_float(v[k]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < S; ++i) h[i] = n + i < N ? p[n + i] : 0.0f;
    }
}
template <int S, bool FULL>
__device__ inline void store_states(float* p, int n, int N, const float* h) {
    if constexpr (FULL) {
#pragma unroll
        for (int i = 0; i < S; i += 4) ((Loose<float>*)(p + n + i))->v = F32::pack(h + i);
    } else {
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (n + i < N) p[n + i] = h[i];
    }
}

// Which batch, run, group and channel a lane works at; the item w of the launch.
template <int L>
struct Place {
    int64_t b, chunk, group, tile;
    uint32_t d;                 // the channel
    int64_t first, end, live;   // the run's tokens, and those of them that the batch has
    int j;                      // which of the channel's lanes
    bool active;
    __device__ Place(const ScanParams& p, int64_t w) {
        constexpr int kChannels = 64 / L;
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        tile = w % p.tiles;
        w /= p.tiles;
        group = w % p.G;
        w /= p.G;
        chunk = w % p.chunks;
        b = w / p.chunks;
        j = lane % L;
        const int64_t c = (tile * kWaves + wave) * kChannels + lane / L;
        active = c < p.Dg;
        d = (uint32_t)(group * p.Dg + (active ? c : 0));
        first = chunk * p.chunk;
        end = min(first + p.chunk, p.T);
        int64_t length = p.T;
        if (p.in.lengths) length = min(max((int64_t)p.in.lengths[b], (int64_t)0), p.T);
        live = max(min(end, length), first);
    }
    // Index of this channel's states within [B][runs][D][N], of run c.
    __device__ int64_t states(const ScanParams& p, int64_t c) const { return ((b * p.chunks + c) * p.D + d) * p.N; }
};

// A tile's rows of B (or C), kTile tokens of NP states from token t on, by the block's
// threads: values in registers, then as floats in LDS.  Zeros past the last token
// that the batch has, and past the N states.
template <class E, int NP>
struct Shared {
    static constexpr int kPer = (kTile * NP + 64 * kWaves - 1) / (64 * kWaves);
    typename E::store v[kPer];
    __device__ void load(const typename E::store* row, int64_t s_t, int64_t t, int64_t live, int N) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = i * 64 * kWaves + threadIdx.x, n = e % NP;
            const int64_t at = t + e / NP;
            v[i] = typename E::store();
            if (e < kTile * NP && n < N && at < live) v[i] = row[at * s_t + n];
        }
    }
    __device__ void store(float* lds) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = i * 64 * kWaves + threadIdx.x;
            if (e < kTile * NP) lds[e] = E::one(v[i]);
        }
    }
};

// The tokens of a tile that are a lane's own, t + k L + j, of its channel d.  (A lane to itself, with 16 tokens,
// keeps no address: the rows' are uniform, the channel's offset has 32 bits.)
template <class E, int L>
struct Own {
    static constexpr int kOwn = kTile / L;
    typename E::store v[kOwn];
    __device__ void load(const typename E::store* rows, int64_t s_t, uint32_t d, int64_t t, int64_t live, bool active,
                         int j) {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const int64_t at = t + k * L + (L == 1 ? 0 : j);
            v[k] = typename E::store();
            if (active && at < live) v[k] = (rows + at * s_t)[d];
        }
    }
};

// Forward over a run: its outputs and states, or (STATES) only the states that it ends
// with from zero, and the sum of its steps.
template <class E, int L, int S, bool FULL, bool STATES>
__global__ __launch_bounds__(64 * kWaves, 2) void swr_scan_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int NP = L * S, OWN = kTile / L;
    __shared__ __attribute__((aligned(16))) float lds_b[2][kTile * NP], lds_c[2][STATES ? 4 : kTile * NP];
    int buf = 0;
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const Place<L> at(p, w);
        const int n0 = at.j * S;
        const T* x = (const T*)p.in.x + at.b * p.sx_b;
        const T* dt = (const T*)p.in.dt + at.b * p.sdt_b;
        const T* z = p.in.z ? (const T*)p.in.z + at.b * p.sz_b : nullptr;
        const T* B = (const T*)p.in.B + at.b * p.sB_b + at.group * p.sB_g;
        const T* C = (const T*)p.in.C + at.b * p.sC_b + at.group * p.sC_g;
        T* y = p.y ? (T*)p.y + at.b * p.sy_b : nullptr;
        const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
        const float skip = p.in.skip ? p.in.skip[at.d] : 0.0f;
        float A[S], h[S];
        load_states<S, FULL>(p.in.A + (int64_t)at.d * p.N, n0, p.N, A);
#pragma unroll
        for (int i = 0; i < S; ++i) {
            A[i] = finite(A[i] * kLog2e);
            h[i] = 0.0f;
        }
        if constexpr (!STATES) {
            if (p.chunks > 1) load_states<S, FULL>(p.states + at.states(p, at.chunk), n0, p.N, h);
            else if (p.in.h0) load_states<S, FULL>(p.in.h0 + (at.b * p.D + at.d) * p.N, n0, p.N, h);
        }
        float steps = 0.0f;
        Own<E, L> rx, rdt, rz;
        Shared<E, NP> rb, rc;
        const auto fetch = [&](int64_t t) {
            rx.load(x, p.sx_t, at.d, t, at.live, at.active, at.j);
            rdt.load(dt, p.sdt_t, at.d, t, at.live, at.active, at.j);
            rb.load(B, p.sB_t, t, at.live, p.N);
            if constexpr (!STATES) {
                if (z) rz.load(z, p.sz_t, at.d, t, at.live, at.active, at.j);
                rc.load(C, p.sC_t, t, at.live, p.N);
            }
        };
        fetch(at.first);
        for (int64_t t = at.first; t < (STATES ? at.live : at.end); t += kTile, buf ^= 1) {
            if constexpr (!STATES)
                if (p.carriers && at.active)
                    store_states<S, FULL>(p.carriers + ((at.b * ((p.T + kTile - 1) / kTile) + t / kTile) * p.D + at.d) *
                                                           p.N, n0, p.N, h);
            float sv[OWN], uv[OWN], xv[OWN], yv[OWN], zv[OWN];
            const auto live = [&](int k) { return t + k * L + (L == 1 ? 0 : at.j) < at.live && at.active; };
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const float v = E::one(rdt.v[k]) + bias;
                sv[k] = p.softplus ? Softplus(v).value : v;
                if (!live(k)) sv[k] = 0.0f;
                xv[k] = E::one(rx.v[k]);
                uv[k] = sv[k] * xv[k];
                yv[k] = 0.0f;
                if constexpr (STATES) steps += sv[k];
                else zv[k] = E::one(rz.v[k]);
            }
            // A token's output, of its sum over the states.
            const auto finish = [&](int k, float sum, float xk, float zk) {
                const int64_t token = t + k * L + (L == 1 ? 0 : at.j);
                float v = fmaf(skip, xk, sum);
                if (z) v *= zk * sigmoid(zk);
                if (y && at.active && token < at.end) (y + token * p.sy_t)[at.d] = E::to(live(k) ? v : 0.0f);
            };
            rb.store(lds_b[buf]);
            if constexpr (!STATES) rc.store(lds_c[buf]);
            fetch(t + kTile);
            __syncthreads();
            each<kTile>([&](auto index) {
                constexpr int tt = index, k = tt / L, jj = tt % L;
                const float s = from_lane<L, jj>(sv[k]), u = from_lane<L, jj>(uv[k]);
                const float* bt = lds_b[buf] + tt * NP + n0;
                const float* ct = lds_c[buf] + (STATES ? 0 : tt * NP + n0);
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    h[i] = fmaf(__builtin_amdgcn_exp2f(s * A[i]), h[i], u * bt[i]);
                    if constexpr (!STATES) {
                        if (FULL || n0 + i < p.N) sum = fmaf(ct[i], h[i], sum);
                    }
                }
                if constexpr (!STATES) {
                    sum = lane_sum<L>(sum);
                    if (L == 1 || at.j == jj) yv[k] = sum;
                    if constexpr (jj == L - 1) finish(k, yv[k], xv[k], zv[k]);
                }
                // (Without it the tile's LDS reads are all brought forward, and spill.)
                if constexpr (S == 16 || tt % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            });
        }
        if constexpr (STATES) {
            steps = lane_sum<L>(steps);
            if (at.active) {
                store_states<S, FULL>(p.states + at.states(p, at.chunk), n0, p.N, h);
                if (at.j == 0) p.steps[(at.b * p.chunks + at.chunk) * p.D + at.d] = steps;
            }
        } else if (p.h_last && at.active && at.chunk == p.chunks - 1) {
            store_states<S, FULL>(p.h_last + (at.b * p.D + at.d) * p.N, n0, p.N, h);
        }
    }
}

// Chains the runs of a state: in place of a run's own states those that it starts from
// (BACK: the gradient that reaches its last states).
template <bool BACK>
__global__ __launch_bounds__(256) void swr_scan_chain_kernel(ScanParams p) {
    const int64_t all = p.B * p.D * p.N, each = p.D * p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t b = i / each, at = i - b * each, d = at / p.N;
        const float rate = finite(p.in.A[at] * kLog2e);
        float h = 0.0f;
        if (BACK ? p.dh_last != nullptr : p.in.h0 != nullptr) h = BACK ? p.dh_last[i] : p.in.h0[i];
        float* s = p.states + b * p.chunks * each + at;
        const float* steps = p.steps + b * p.chunks * p.D + d;
        // (The last run of the order has no run after it, and its own states were not taken.)
#pragma unroll 8
        for (int64_t k = 0; k + 1 < p.chunks; ++k) {
            const int64_t c = BACK ? p.chunks - 1 - k : k;
            const float own = s[c * each], total = steps[c * p.D];
            s[c * each] = h;
            h = fmaf(__builtin_amdgcn_exp2f(rate * total), h, own);
        }
        s[BACK ? 0 : (p.chunks - 1) * each] = h;
    }
}

// A few tokens: no tiles, nothing shared, a token after the other; the states move once.
template <class E, int L, bool FULL>
__global__ __launch_bounds__(64 * kWaves) void swr_scan_step_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int S = 4;
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const Place<L> at(p, w);
        if (!at.active) continue;
        const int n0 = at.j * S;
        const int64_t own = (at.b * p.D + at.d) * p.N;
        const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
        const float skip = p.in.skip ? p.in.skip[at.d] : 0.0f;
        float A[S], h[S] = {};
        load_states<S, FULL>(p.in.A + (int64_t)at.d * p.N, n0, p.N, A);
        if (p.in.h0) load_states<S, FULL>(p.in.h0 + own, n0, p.N, h);
#pragma unroll
        for (int i = 0; i < S; ++i) A[i] = finite(A[i] * kLog2e);
        if (p.carriers) store_states<S, FULL>(p.carriers + own, n0, p.N, h);   // (a single block of tokens)
        for (int64_t t = 0; t < at.end; ++t) {
            float v = 0.0f;
            if (t < at.live) {
                const T* bt = (const T*)p.in.B + at.b * p.sB_b + t * p.sB_t + at.group * p.sB_g;
                const T* ct = (const T*)p.in.C + at.b * p.sC_b + t * p.sC_t + at.group * p.sC_g;
                const float x = E::one(((const T*)p.in.x)[at.b * p.sx_b + t * p.sx_t + at.d]);
                float s = E::one(((const T*)p.in.dt)[at.b * p.sdt_b + t * p.sdt_t + at.d]) + bias;
                float z = 0.0f;
                if (p.in.z) z = E::one(((const T*)p.in.z)[at.b * p.sz_b + t * p.sz_t + at.d]);
                float bv[S], cv[S];
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    bv[i] = FULL || n0 + i < p.N ? E::one(bt[n0 + i]) : 0.0f;
                    cv[i] = FULL || n0 + i < p.N ? E::one(ct[n0 + i]) : 0.0f;
                }
                if (p.softplus) s = Softplus(s).value;
                const float u = s * x;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    h[i] = fmaf(__builtin_amdgcn_exp2f(s * A[i]), h[i], u * bv[i]);
                    if (FULL || n0 + i < p.N) v = fmaf(cv[i], h[i], v);
                }
                v = fmaf(skip, x, lane_sum<L>(v));
                if (p.in.z) v *= z * sigmoid(z);
            }
            if (p.y && at.j == 0) ((T*)p.y)[at.b * p.sy_b + t * p.sy_t + at.d] = E::to(v);
        }
        if (p.h_last) store_states<S, FULL>(p.h_last + own, n0, p.N, h);
    }
}

// What the backward takes of a lane's own tokens.
template <class E, int L>
struct OwnGradients {
    Own<E, L> x, dt, z, dy;
};

// Backward over a run from its end: the gradient that leaves it to the run before, from
// zero, and the sum of its steps.
template <class E, int L, int S, bool FULL>
__global__ __launch_bounds__(64 * kWaves, 2) void swr_scan_back_states_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int NP = L * S, OWN = kTile / L;
    __shared__ __attribute__((aligned(16))) float lds_c[2][kTile * NP];
    int buf = 0;
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const Place<L> at(p, w);
        const int n0 = at.j * S;
        const T* dt = (const T*)p.in.dt + at.b * p.sdt_b;
        const T* z = p.in.z ? (const T*)p.in.z + at.b * p.sz_b : nullptr;
        const T* dy = (const T*)p.dy + at.b * p.sy_b;
        const T* C = (const T*)p.in.C + at.b * p.sC_b + at.group * p.sC_g;
        const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
        float A[S], g[S];
        load_states<S, FULL>(p.in.A + (int64_t)at.d * p.N, n0, p.N, A);
#pragma unroll
        for (int i = 0; i < S; ++i) {
            A[i] = finite(A[i] * kLog2e);
            g[i] = 0.0f;
        }
        float steps = 0.0f;
        Own<E, L> rdt, rz, rdy;
        Shared<E, NP> rc;
        const auto fetch = [&](int64_t t) {
            if (t < at.first) return;
            rdt.load(dt, p.sdt_t, at.d, t, at.live, at.active, at.j);
            if (z) rz.load(z, p.sz_t, at.d, t, at.live, at.active, at.j);
            rdy.load(dy, p.sy_t, at.d, t, at.live, at.active, at.j);
            rc.load(C, p.sC_t, t, at.live, p.N);
        };
        const int64_t last = at.first + (at.live - at.first + kTile - 1) / kTile * kTile - kTile;
        fetch(last);
        for (int64_t t = last; t >= at.first; t -= kTile, buf ^= 1) {
            float sv[OWN], wv[OWN];
            const auto live = [&](int k) { return t + k * L + (L == 1 ? 0 : at.j) < at.live && at.active; };
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const float v = E::one(rdt.v[k]) + bias;
                sv[k] = p.softplus ? Softplus(v).value : v;
                if (!live(k)) sv[k] = 0.0f;
                steps += sv[k];
                wv[k] = E::one(rdy.v[k]);
                if (z) {
                    const float zk = E::one(rz.v[k]);
                    wv[k] *= zk * sigmoid(zk);
                }
            }
            rc.store(lds_c[buf]);
            fetch(t - kTile);
            __syncthreads();
            each<kTile>([&](auto index) {
                constexpr int tt = kTile - 1 - index, k = tt / L, jj = tt % L;
                const float s = from_lane<L, jj>(sv[k]), u = from_lane<L, jj>(wv[k]);
                const float* ct = lds_c[buf] + tt * NP + n0;
#pragma unroll
                for (int i = 0; i < S; ++i) g[i] = __builtin_amdgcn_exp2f(s * A[i]) * fmaf(ct[i], u, g[i]);
            });
        }
        steps = lane_sum<L>(steps);
        if (at.active) {
            store_states<S, FULL>(p.states + at.states(p, at.chunk), n0, p.N, g);
            if (at.j == 0) p.steps[(at.b * p.chunks + at.chunk) * p.D + at.d] = steps;
        }
    }
}

// Sums of four values over a wave's channels: of every value, over the lanes that have the
// same place among their channel's L.  A swap of a register's halves with another's takes
// two values to the sums of each in half the lanes; the lane of row r (of 16 lanes) ends up
// with the value of index value_of_row(r), the same at every place mod L.
template <int L>
__device__ inline float channel_sums(const float* v) {
    const auto halves = [](float a, float b) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                                        false, false);
        return as_float(r[0]) + as_float(r[1]);
    };
    const auto rows = [](float a, float b) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                                        false, false);
        return as_float(r[0]) + as_float(r[1]);
    };
    float s = rows(halves(v[0], v[1]), halves(v[2], v[3]));
    if constexpr (L <= 8) s += dpp<kRotate8>(s);
    if constexpr (L <= 4) s += dpp<kRotate4>(s);
    if constexpr (L <= 2) s += dpp<kXor2>(s);
    if constexpr (L <= 1) s += dpp<kXor1>(s);
    return s;
}
__device__ inline int value_of_row(int row) { return row == 1 ? 2 : row == 2 ? 1 : row; }

// Backward over a run, tile by tile from its end: a tile's states anew from its carriers, kept
// with their decays in registers (4 states a lane, 16 tokens), then the tokens from the last.
template <class E, int L, bool FULL>
__global__ __launch_bounds__(64 * kWaves, 1) void swr_scan_back_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int S = 4, NP = L * S, OWN = kTile / L;
    __shared__ __attribute__((aligned(16))) float lds_b[2][kTile * NP], lds_c[2][kTile * NP];
    __shared__ float lds_sum[kWaves][kTile][2][NP];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int buf = 0;
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const Place<L> at(p, w);
        const int n0 = at.j * S;
        const T* x = (const T*)p.in.x + at.b * p.sx_b;
        const T* dt = (const T*)p.in.dt + at.b * p.sdt_b;
        const T* z = p.in.z ? (const T*)p.in.z + at.b * p.sz_b : nullptr;
        const T* dy = (const T*)p.dy + at.b * p.sy_b;
        const T* B = (const T*)p.in.B + at.b * p.sB_b + at.group * p.sB_g;
        const T* C = (const T*)p.in.C + at.b * p.sC_b + at.group * p.sC_g;
        const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
        const float skip = p.in.skip ? p.in.skip[at.d] : 0.0f;
        float A[S], g[S] = {}, dA[S] = {}, dbias = 0.0f, dskip = 0.0f;
        load_states<S, FULL>(p.in.A + (int64_t)at.d * p.N, n0, p.N, A);
#pragma unroll
        for (int i = 0; i < S; ++i) A[i] = finite(A[i]);
        if (p.chunks > 1) load_states<S, FULL>(p.states + at.states(p, at.chunk), n0, p.N, g);
        else if (p.dh_last) load_states<S, FULL>(p.dh_last + (at.b * p.D + at.d) * p.N, n0, p.N, g);
        if (!at.active) {
#pragma unroll
            for (int i = 0; i < S; ++i) g[i] = 0.0f;   // (it takes part in the sums over channels)
        }
        OwnGradients<E, L> raw;
        Shared<E, NP> rb, rc;
        float start[S];
        const auto fetch = [&](int64_t t) {
            if (t < at.first || t >= at.live) return;
            raw.x.load(x, p.sx_t, at.d, t, at.live, at.active, at.j);
            raw.dt.load(dt, p.sdt_t, at.d, t, at.live, at.active, at.j);
            if (z) raw.z.load(z, p.sz_t, at.d, t, at.live, at.active, at.j);
            raw.dy.load(dy, p.sy_t, at.d, t, at.live, at.active, at.j);
            rb.load(B, p.sB_t, t, at.live, p.N);
            rc.load(C, p.sC_t, t, at.live, p.N);
            load_states<S, FULL>(p.carriers_in + ((at.b * ((p.T + kTile - 1) / kTile) + t / kTile) * p.D + at.d) * p.N,
                                 n0, p.N, start);
        };
        const int64_t last = at.first + (at.end - at.first + kTile - 1) / kTile * kTile - kTile;
        fetch(last);
        for (int64_t t = last; t >= at.first; t -= kTile) {
            const int64_t tokens = min((int64_t)kTile, at.end - t);
            T* dx = (T*)p.out.dx + (at.b * p.T + t) * p.D + at.d;
            T* ddt = (T*)p.out.ddt + (at.b * p.T + t) * p.D + at.d;
            T* dz = z ? (T*)p.out.dz + (at.b * p.T + t) * p.D + at.d : nullptr;
            float* shares = p.shares + (((at.b * p.T + t) * p.G + at.group) * p.tiles + at.tile) * 2 * p.N;
            const int64_t step = p.G * p.tiles * 2 * p.N;   // of the shares, from token to token
            if (t >= at.live) {   // past the batch's last token
                if (at.active) {
#pragma unroll
                    for (int k = 0; k < OWN; ++k) {
                        const int64_t tt = k * L + at.j;
                        if (tt < tokens) {
                            dx[tt * p.D] = ddt[tt * p.D] = E::to(0.0f);
                            if (z) dz[tt * p.D] = E::to(0.0f);
                        }
                    }
                }
                for (int e = threadIdx.x; e < kTile * 2 * NP; e += 64 * kWaves) {
                    const int tt = e / (2 * NP), which = e / NP % 2, n = e % NP;
                    if (tt < tokens && n < p.N) shares[tt * step + which * p.N + n] = 0.0f;
                }
                fetch(t - kTile);
                continue;
            }
            const auto live = [&](int k) { return t + k * L + (L == 1 ? 0 : at.j) < at.live && at.active; };
            float sv[OWN], slope[OWN], uv[OWN], xv[OWN], wv[OWN], zv[OWN], dyv[OWN], yv[OWN], s1[OWN], s2[OWN];
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const float v = E::one(raw.dt.v[k]) + bias;
                sv[k] = v;
                slope[k] = 1.0f;
                if (p.softplus) {
                    const Softplus s(v);
                    sv[k] = s.value;
                    slope[k] = s.slope;
                }
                if (!live(k)) sv[k] = 0.0f;
                xv[k] = E::one(raw.x.v[k]);
                uv[k] = sv[k] * xv[k];
                wv[k] = dyv[k] = E::one(raw.dy.v[k]);
                if (z) {
                    zv[k] = E::one(raw.z.v[k]);
                    wv[k] *= zv[k] * sigmoid(zv[k]);
                }
                yv[k] = s1[k] = s2[k] = 0.0f;
            }
            float a[kTile][S], h[kTile + 1][S];
#pragma unroll
            for (int i = 0; i < S; ++i) h[0][i] = at.active ? start[i] : 0.0f;
            rb.store(lds_b[buf]);
            rc.store(lds_c[buf]);
            fetch(t - kTile);
            __syncthreads();
            each<kTile>([&](auto index) {
                constexpr int tt = index, k = tt / L, jj = tt % L;
                const float s = from_lane<L, jj>(sv[k]) * kLog2e, u = from_lane<L, jj>(uv[k]);
                const float* bt = lds_b[buf] + tt * NP + n0;
                const float* ct = lds_c[buf] + tt * NP + n0;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    a[tt][i] = __builtin_amdgcn_exp2f(s * A[i]);
                    h[tt + 1][i] = fmaf(a[tt][i], h[tt][i], u * bt[i]);
                    sum = fmaf(ct[i], h[tt + 1][i], sum);
                }
                if (z) {
                    sum = lane_sum<L>(sum);
                    if (L == 1 || at.j == jj) yv[k] = sum;
                }
            });
            each<kTile>([&](auto index) {
                constexpr int tt = kTile - 1 - index, k = tt / L, jj = tt % L;
                const float s = from_lane<L, jj>(sv[k]), u = from_lane<L, jj>(uv[k]), wt = from_lane<L, jj>(wv[k]);
                const float* bt = lds_b[buf] + tt * NP + n0;
                const float* ct = lds_c[buf] + tt * NP + n0;
                float db[S], dc[S], along = 0.0f, decay = 0.0f;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    g[i] = fmaf(ct[i], wt, g[i]);
                    dc[i] = h[tt + 1][i] * wt;
                    db[i] = g[i] * u;
                    along = fmaf(g[i], bt[i], along);
                    g[i] *= a[tt][i];
                    const float past = g[i] * h[tt][i];
                    decay = fmaf(past, A[i], decay);
                    dA[i] = fmaf(past, s, dA[i]);
                }
                const float sb = channel_sums<L>(db), sc = channel_sums<L>(dc);
                if (lane % 16 < L) {
                    const int n = (lane % 16) * S + value_of_row(lane / 16);
                    lds_sum[wave][tt][0][n] = sb;
                    lds_sum[wave][tt][1][n] = sc;
                }
                along = lane_sum<L>(along);
                decay = lane_sum<L>(decay);
                if (L == 1 || at.j == jj) {
                    s1[k] = along;
                    s2[k] = decay;
                }
            });
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const int64_t tt = k * L + at.j;
                const bool has = live(k);
                const float v = has ? fmaf(xv[k], s1[k], s2[k]) * slope[k] : 0.0f;
                dbias += v;
                dskip = fmaf(wv[k], xv[k], dskip);
                if (at.active && tt < tokens) {
                    dx[tt * p.D] = E::to(has ? fmaf(sv[k], s1[k], skip * wv[k]) : 0.0f);
                    ddt[tt * p.D] = E::to(v);
                    if (z) {
                        const float gate = sigmoid(zv[k]);
                        const float f = dyv[k] * fmaf(skip, xv[k], yv[k]) * (gate * fmaf(zv[k], 1.0f - gate, 1.0f));
                        dz[tt * p.D] = E::to(has ? f : 0.0f);
                    }
                }
            }
            __syncthreads();
            for (int e = threadIdx.x; e < kTile * 2 * NP; e += 64 * kWaves) {
                const int tt = e / (2 * NP), which = e / NP % 2, n = e % NP;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < kWaves; ++i) sum += lds_sum[i][tt][which][n];
                if (tt < tokens && n < p.N) shares[tt * step + which * p.N + n] = sum;
            }
            buf ^= 1;
        }
        dbias = lane_sum<L>(dbias);
        dskip = lane_sum<L>(dskip);
        if (at.active) {
            float* sums = p.sums + ((at.b * p.chunks + at.chunk) * p.D + at.d) * (p.N + 2);
            store_states<S, FULL>(sums, n0, p.N, dA);
            if (at.j == 0) {
                sums[p.N] = dbias;
                sums[p.N + 1] = dskip;
            }
            if (p.out.dh0 && at.chunk == 0)
                store_states<S, FULL>(p.out.dh0 + (at.b * p.D + at.d) * p.N, n0, p.N, g);
        }
    }
}

// dB and dC from the shares of a group's blocks of channels.
template <class E>
__global__ __launch_bounds__(256) void swr_scan_join_kernel(ScanParams p) {
    typedef typename E::store T;
    const int64_t rows = p.B * p.T * p.G, all = rows * 2 * p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / (2 * p.N);
        const int at = (int)(i - row * 2 * p.N), which = at >= p.N;
        const float* s = p.shares + row * p.tiles * 2 * p.N + at;
        float sum = 0.0f;
#pragma unroll 8
        for (int64_t k = 0; k < p.tiles; ++k) sum += s[k * 2 * p.N];
        ((T*)(which ? p.out.dC : p.out.dB))[row * p.N + at - which * p.N] = E::to(sum);
    }
}

// dA, dbias and dskip from the runs' shares.
__global__ __launch_bounds__(256) void swr_scan_sums_kernel(ScanParams p) {
    const int64_t each = p.D * (p.N + 2), runs = p.B * p.chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < each; i += (int64_t)gridDim.x * 256) {
        const int64_t d = i / (p.N + 2);
        const int n = (int)(i - d * (p.N + 2));
        float sum = 0.0f;
#pragma unroll 8
        for (int64_t k = 0; k < runs; ++k) sum += p.sums[k * each + i];
        if (n < p.N) p.out.dA[d * p.N + n] = sum;
        else if (n == p.N) { if (p.out.dbias) p.out.dbias[d] = sum; }
        else if (p.out.dskip) p.out.dskip[d] = sum;
    }
}

constexpr int64_t kMostBlocks = 1 << 20;
constexpr int64_t kFew = 8;   // tokens that the step kernel takes

unsigned grid_of(int64_t blocks) { return (unsigned)std::max<int64_t>(1, std::min(blocks, kMostBlocks)); }

// f<L, S, FULL>(): the kernels of a plan.
template <class F>
hipError_t narrow(const ScanPlan& plan, int N, F f) {
    const bool full = N == 4 * plan.lanes;
    switch (plan.lanes) {
        case 1: return full ? f.template operator()<1, 4, true>() : f.template operator()<1, 4, false>();
        case 2: return full ? f.template operator()<2, 4, true>() : f.template operator()<2, 4, false>();
        case 4: return full ? f.template operator()<4, 4, true>() : f.template operator()<4, 4, false>();
        case 8: return full ? f.template operator()<8, 4, true>() : f.template operator()<8, 4, false>();
        case 16: return full ? f.template operator()<16, 4, true>() : f.template operator()<16, 4, false>();
    }
    return hipErrorInvalidValue;
}
template <class F>
hipError_t wide(const ScanPlan& plan, F f) {
    switch (plan.lanes) {
        case 1: return f.template operator()<1, 16, true>();
        case 2: return f.template operator()<2, 16, true>();
        case 4: return f.template operator()<4, 16, true>();
    }
    return hipErrorInvalidValue;
}

template <class E, bool STATES>
struct Forward {
    const ScanParams& p;
    hipStream_t st;
    template <int L, int S, bool FULL>
    hipError_t operator()() const {
        hipLaunchKernelGGL((swr_scan_kernel<E, L, S, FULL, STATES>), dim3(grid_of(p.work)), dim3(64 * kWaves), 0, st, p);
        return hipGetLastError();
    }
};
template <class E>
struct Step {
    const ScanParams& p;
    hipStream_t st;
    template <int L, int S, bool FULL>
    hipError_t operator()() const {
        hipLaunchKernelGGL((swr_scan_step_kernel<E, L, FULL>), dim3(grid_of(p.work)), dim3(64 * kWaves), 0, st, p);
        return hipGetLastError();
    }
};
template <class E>
struct BackStates {
    const ScanParams& p;
    hipStream_t st;
    template <int L, int S, bool FULL>
    hipError_t operator()() const {
        hipLaunchKernelGGL((swr_scan_back_states_kernel<E, L, S, FULL>), dim3(grid_of(p.work)), dim3(64 * kWaves), 0, st,
                           p);
        return hipGetLastError();
    }
};
template <class E>
struct Back {
    const ScanParams& p;
    hipStream_t st;
    template <int L, int S, bool FULL>
    hipError_t operator()() const {
        hipLaunchKernelGGL((swr_scan_back_kernel<E, L, FULL>), dim3(grid_of(p.work)), dim3(64 * kWaves), 0, st, p);
        return hipGetLastError();
    }
};

template <class E>
hipError_t forward(const ScanPlan& plan, const ScanParams& p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (p.T <= kFew) return narrow(plan, p.N, Step<E>{p, st});
    if (plan.chunks > 1) {
        const Forward<E, true> states{p, st};
        if ((e = plan.wide ? wide(plan, states) : narrow(plan, p.N, states)) != hipSuccess) return e;
        hipLaunchKernelGGL(swr_scan_chain_kernel<false>, dim3(grid_of((p.B * p.D * p.N + 255) / 256)), dim3(256), 0, st,
                           p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const Forward<E, false> all{p, st};
    return plan.wide ? wide(plan, all) : narrow(plan, p.N, all);
}

template <class E>
hipError_t backward(const ScanPlan& plan, const ScanParams& p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (plan.chunks > 1) {
        if ((e = narrow(plan, p.N, BackStates<E>{p, st})) != hipSuccess) return e;
        hipLaunchKernelGGL(swr_scan_chain_kernel<true>, dim3(grid_of((p.B * p.D * p.N + 255) / 256)), dim3(256), 0, st,
                           p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if ((e = narrow(plan, p.N, Back<E>{p, st})) != hipSuccess) return e;
    hipLaunchKernelGGL(swr_scan_join_kernel<E>, dim3(grid_of((p.B * p.T * p.G * 2 * p.N + 255) / 256)), dim3(256), 0, st,
                       p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(swr_scan_sums_kernel, dim3(grid_of((p.D * (p.N + 2) + 255) / 256)), dim3(256), 0, st, p);
    return hipGetLastError();
}

int lanes_of(int N, int states) {
    int lanes = 1;
    while (lanes * states < N) lanes *= 2;
    return lanes;
}

}  // namespace

ScanPlan plan_scan(const swr_scan_t& p, bool backward) {
    const int64_t dg = p.D / p.G, kWant = 512;
    const auto make = [&](bool wide) {
        ScanPlan plan = {};
        plan.wide = wide;
        plan.lanes = lanes_of(p.N, wide ? 16 : 4);
        const int64_t channels = kWaves * (64 / plan.lanes);
        plan.tiles = (dg + channels - 1) / channels;
        plan.chunks = 1;
        plan.chunk = std::max<int64_t>(kTile, (p.T + kTile - 1) / kTile * kTile);
        return plan;
    };
    ScanPlan plan = make(false);
    if (p.T <= kFew && !backward) return plan;
    const bool can = !backward && (p.N == 16 || p.N == 32 || p.N == 64);
    const int64_t blocks = plan.blocks(p.B, p.G);
    if (can && (make(true).blocks(p.B, p.G) >= kWant || blocks < kWant)) plan = make(true);
    // Runs of at least 64 tokens, as many as fill the GPU.
    const int64_t one = std::max<int64_t>(1, plan.blocks(p.B, p.G));   // (a batch of none has none)
    const int64_t most = std::max<int64_t>(1, p.T / 64);
    const int64_t chunks = std::min(most, (kWant + one - 1) / one);
    if (one < kWant && chunks > 1) {
        plan.chunk = ((p.T + chunks - 1) / chunks + kTile - 1) / kTile * kTile;
        plan.chunks = (p.T + plan.chunk - 1) / plan.chunk;
    }
    return plan;
}

int64_t scan_work_floats(const swr_scan_t& p, const ScanPlan& plan) {
    return plan.chunks > 1 ? p.B * plan.chunks * p.D * (p.N + 1) : 0;
}

int64_t scan_backward_work_floats(const swr_scan_t& p, const ScanPlan& plan) {
    return scan_work_floats(p, plan) + p.B * p.T * p.G * plan.tiles * 2 * p.N + p.B * plan.chunks * p.D * (p.N + 2);
}

hipError_t launch_scan(int dtype, const ScanPlan& plan, const ScanParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    return dtype == SWR_DTYPE_F32 ? forward<F32>(plan, p, st) : forward<Bf16>(plan, p, st);
}

hipError_t launch_scan_backward(int dtype, const ScanPlan& plan, const ScanParams& p, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    return dtype == SWR_DTYPE_F32 ? backward<F32>(plan, p, st) : backward<Bf16>(plan, p, st);
}

}  // namespace swr
