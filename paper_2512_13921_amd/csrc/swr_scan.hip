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
// exponential (half the rate), two products and two multiply-adds, 24
// cycles of a SIMD for a wave's 64 states.  16387 tokens of 4096 channels with 16 states take 490 us, which is 72 cycles
// with the helpers' share; 2 x 2048 tokens 127 forward and 370 backward; one more token of 128 requests 17.4, at 4.1 TB/s.
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
template <int L, int WAVES = kWaves>
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
        // Blocks go to the 8 dies in turn, each with an L2 of its own: a die gets a run of channels, whose rows
        // share cache lines.
        if (p.tiles % 8 == 0) tile = tile % 8 * (p.tiles / 8) + tile / 8;
        group = w % p.G;
        w /= p.G;
        chunk = w % p.chunks;
        b = w / p.chunks;
        j = lane % L;
        const int64_t c = (tile * WAVES + wave) * kChannels + lane / L;
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
                if constexpr (tt % 4 == 3) __builtin_amdgcn_sched_barrier(0);
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

// A state a lane: a channel has one row of 16 lanes (two or four for more states), and its tile of 16 tokens
// one token a lane of a row, whose step and input the others take as a row's broadcast.
constexpr int kPad = kTile + 4;   // floats of a state's tile in LDS: 16-byte reads of 16 states meet no bank twice

// Sums over a row's lanes of 16 values: lane l gets that of value l.  Each exchange halves the values:
// a lane keeps those of its half and gets its partner's share of them (partners 8, 7, 2 and 1 apart by bits).
__device__ inline float row_sums(const float* p) {
    const int lane = threadIdx.x;
    float a[8], b[4], c[2];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float keep = lane & 8 ? p[k + 8] : p[k], send = lane & 8 ? p[k] : p[k + 8];
        a[k] = keep + dpp<kRotate8>(send);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float keep = lane & 4 ? a[k + 4] : a[k], send = lane & 4 ? a[k] : a[k + 4];
        b[k] = keep + dpp<kHalfMirror>(send);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float keep = lane & 2 ? b[k + 2] : b[k], send = lane & 2 ? b[k] : b[k + 2];
        c[k] = keep + dpp<kXor2>(send);
    }
    const float keep = lane & 1 ? c[1] : c[0], send = lane & 1 ? c[0] : c[1];
    return keep + dpp<kXor1>(send);
}
__device__ inline float swap_sum16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false,
                                                    false);
    return as_float(r[0]) + as_float(r[1]);
}
__device__ inline float swap_sum32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false,
                                                    false);
    return as_float(r[0]) + as_float(r[1]);
}
// ... and over a channel's R rows.
template <int R>
__device__ inline float state_sums(const float* p) {
    float v = row_sums(p);
    if constexpr (R >= 2) v = swap_sum16(v, v);
    if constexpr (R >= 4) v = swap_sum32(v, v);
    return v;
}
// v of the lane tt of a row.
template <int TT>
__device__ inline float of_token(float v) { return dpp<0x150 + TT>(v); }

// A tile of B (or C) as Shared, in LDS state by state; `last` is the last token that may be read.
template <class E, int NP, int WAVES>
struct SharedRows {
    static constexpr int kAll = kTile * NP, kThreads = 64 * WAVES, kPer = (kAll + kThreads - 1) / kThreads;
    typename E::store v[kPer];
    __device__ void load(const typename E::store* row, int64_t s_t, int64_t t, int64_t last, int N) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = i * kThreads + threadIdx.x % kThreads;
            v[i] = row[min(t + e / NP % kTile, last) * s_t + min(e % NP, N - 1)];
        }
    }
    __device__ void store(float* lds, int64_t tokens, int N) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = i * kThreads + threadIdx.x % kThreads;
            if (kAll % kThreads == 0 || e < kAll)
                lds[e % NP * kPad + e / NP] = e % NP < N && e / NP < tokens ? E::one(v[i]) : 0.0f;
        }
    }
};
// A state's tile.
__device__ inline void read_tile(const float* lds, float* f) {
#pragma unroll
    for (int k = 0; k < kTile; k += 4) {
        const float4 v = *(const float4*)(lds + k);
        f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
    }
}

// Two kinds of waves: four that keep states and work through the tokens, and two helpers for each of them that
// load and prepare its tokens, every second tile each, and finish their outputs.  (A wave alone on its SIMD issues
// an instruction every 6 to 9 cycles, three together one every 4: a sequence of 4096 channels of 16 states,
// one wave of states for each SIMD, took 768 us where a wave did all of it, 731 with one helper.)
//
// Loads, stores and what a token has to itself go by another order of the lanes: tokens, and for
// each the wave's CH channels next to each other, so that lanes next to each other share a cache line.
template <int R>
struct Lanes {
    static constexpr int CH = 4 / R;   // channels of a wave
    int token, channel, part;          // part: which of the channel's R rows' sums is the lane's
    __device__ Lanes() {
        const int lane = threadIdx.x % 64;
        channel = lane % CH;
        token = lane / CH % kTile;
        part = lane / (CH * kTile);
    }
};

// A tensor's rows of a batch, token by token, as buffers: a tile's begins at its first token, and what
// lies past the last element of the last token that may be read (or written) is not: reads give zero.
typedef __amdgpu_buffer_rsrc_t Buffer;
struct Rows {
    const char* base;
    int64_t step;       // bytes from token to token
    int64_t last;       // bytes up to the end of the last token's row
    template <class T>
    __device__ Rows(const T* p, int64_t s_t, int last_token, int64_t width)
        : base((const char*)p), step(s_t * (int64_t)sizeof(T)), last(last_token * step + width * (int64_t)sizeof(T)) {}
    __device__ Buffer from(int t) const {
        const int64_t left = max(last - t * step, (int64_t)0);
        return __builtin_amdgcn_make_buffer_rsrc((void*)(base + t * step), 0, (int)min(left, (int64_t)0x7fffffff),
                                                 0x00027000);
    }
};
template <class T>
__device__ inline T buffer_load(Buffer b, uint32_t bytes) {
    if constexpr (sizeof(T) == 2) return (T)__builtin_amdgcn_raw_buffer_load_b16(b, (int)bytes, 0, 0);
    else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(b, (int)bytes, 0, 0));
}
template <class T>
__device__ inline void buffer_store(T v, Buffer b, uint32_t bytes) {
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(v, b, (int)bytes, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), b, (int)bytes, 0, 0);
}

// Where a lane works (as Place), in both orders of the lanes.  Lanes past the last channel do what the last one's
// do, and store the same values.
template <int R>
struct RowPlace {
    int64_t b, chunk, group;
    int64_t d;                  // the channel whose token the lane loads
    int64_t row_d;              // the channel that its state belongs to
    int n;                      // its state
    int first, end, live;
    __device__ RowPlace(const ScanParams& p, const Lanes<R>& lanes, int64_t w) {
        const Place<16 * R> at(p, w);
        b = at.b; chunk = at.chunk; group = at.group;
        first = (int)at.first; end = (int)at.end;
        live = __builtin_amdgcn_readfirstlane((int)at.live);
        n = at.j;
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % kWaves;
        const int64_t base = (at.tile * kWaves + wave) * Lanes<R>::CH, last = p.Dg - 1;
        d = group * p.Dg + min(base + lanes.channel, last);
        row_d = group * p.Dg + min(base + (int64_t)lane / (16 * R), last);
    }
    __device__ int64_t state(const ScanParams& p) const { return (b * p.D + row_d) * p.N + n; }
    __device__ int64_t run(const ScanParams& p) const { return ((b * p.chunks + chunk) * p.D + row_d) * p.N + n; }
};

// A tile of B (or C) as Shared, in LDS state by state, by WAVES waves.
template <class E, int NP, int WAVES, bool FULL>
struct RowsShared {
    typedef typename E::store T;
    static constexpr int kAll = kTile * NP, kThreads = 64 * WAVES, kPer = (kAll + kThreads - 1) / kThreads;
    T v[kPer];
    // Bytes from a tile's first element to a thread's.
    static __device__ void offsets(int64_t step, int N, uint32_t* at) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = i * kThreads + threadIdx.x % kThreads;
            at[i] = (uint32_t)(e / NP % kTile * step) + (uint32_t)(min(e % NP, N - 1) * (int)sizeof(T));
        }
    }
    __device__ void load(Buffer b, const uint32_t* at, uint32_t more) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = buffer_load<T>(b, at[i] + more);
    }
    __device__ void store(float* lds, int N) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = i * kThreads + threadIdx.x % kThreads;
            if (kAll % kThreads == 0 || e < kAll) lds[e % NP * kPad + e / NP] = FULL || e % NP < N ? E::one(v[i]) : 0.0f;
        }
    }
};

// A lane's products of a tile, in LDS for sums over the states: 16-byte writes by lane and reads by
// token, without bank conflicts either way.
constexpr int kProducts = 64 * kPad + 64;
__device__ inline int product_at(int lane) { return lane * kPad + lane / 16 * 16; }

// As swr_scan_kernel, a state a lane.
template <class E, int R, bool FULL, bool STATES, bool CARRY>
__global__ __launch_bounds__(192 * kWaves, R == 1 ? 6 : 3) void swr_scan_rows_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int NP = 16 * R;
    constexpr int kRound = 4;   // tiles of a round, two for each helper; loads go as far ahead
    __shared__ __attribute__((aligned(16))) float lds_b[kRound][NP * kPad], lds_c[kRound][STATES ? 4 : NP * kPad];
    __shared__ float lds_s[kRound][kWaves][64], lds_u[kRound][kWaves][64];
    __shared__ __attribute__((aligned(16))) float lds_p[2][kWaves][STATES ? 4 : kProducts];
    const Lanes<R> lanes;
    const int lane = threadIdx.x % 64, place = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int wave = place % kWaves, helper = place / kWaves - 1;   // helpers 0 and 1; -1: states
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const RowPlace<R> at(p, lanes, w);
        // (Whole rounds: the last tiles may have no token, and change nothing.)
        const int tiles = (at.live - at.first + kRound * kTile - 1) / (kRound * kTile) * kRound;
        if (helper >= 0) {
            const int last = at.live - 1;
            const Rows x((const T*)p.in.x + at.b * p.sx_b, p.sx_t, last, p.D);
            const Rows dt((const T*)p.in.dt + at.b * p.sdt_b, p.sdt_t, last, p.D);
            const Rows z(p.in.z ? (const T*)p.in.z + at.b * p.sz_b : (const T*)p.in.x + at.b * p.sx_b,
                         p.in.z ? p.sz_t : p.sx_t, last, p.D);
            const Rows B((const T*)p.in.B + at.b * p.sB_b + at.group * p.sB_g, p.sB_t, last, p.N);
            const Rows C((const T*)p.in.C + at.b * p.sC_b + at.group * p.sC_g, p.sC_t, last, p.N);
            const Rows y((const T*)p.y + at.b * p.sy_b, p.sy_t, at.end - 1, p.D);
            typedef RowsShared<E, NP, kWaves, FULL> Parts;
            const uint32_t channel = (uint32_t)(at.d * (int64_t)sizeof(T));
            const uint32_t at_x = (uint32_t)(lanes.token * x.step) + channel, at_dt = (uint32_t)(lanes.token * dt.step) + channel;
            const uint32_t at_z = (uint32_t)(lanes.token * z.step) + channel, at_y = (uint32_t)(lanes.token * y.step) + channel;
            uint32_t at_b[Parts::kPer], at_c[Parts::kPer];
            Parts::offsets(B.step, p.N, at_b);
            Parts::offsets(C.step, p.N, at_c);
            const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
            const float skip = p.in.skip ? p.in.skip[at.d] : 0.0f;
            struct Raw {
                T x, dt, z;
                Parts b, c;
            } raw[2];
            struct Streams {   // from a token on
                Buffer x, dt, z, b, c;
            };
            const auto from = [&](int t) { return Streams{x.from(t), dt.from(t), z.from(t), B.from(t), C.from(t)}; };
            const auto fetch = [&](Raw& r, const Streams& from, int tokens) {
                r.x = buffer_load<T>(from.x, at_x + (uint32_t)(tokens * (int)x.step));
                r.dt = buffer_load<T>(from.dt, at_dt + (uint32_t)(tokens * (int)dt.step));
                if constexpr (!STATES) r.z = buffer_load<T>(from.z, at_z + (uint32_t)(tokens * (int)z.step));
                r.b.load(from.b, at_b, (uint32_t)(tokens * (int)B.step));
                if constexpr (!STATES) r.c.load(from.c, at_c, (uint32_t)(tokens * (int)C.step));
            };
            float steps = 0.0f;
            const auto prepare = [&](Raw& r, int t, float& xv, float& zv, int second) {
                const int slot = helper + 2 * second;
                const float v = E::one(r.dt) + bias;
                float sv = p.softplus ? Softplus(v).value : v;
                sv = t + lanes.token < at.live ? sv : 0.0f;
                xv = t + lanes.token < at.live ? E::one(r.x) : 0.0f;
                if constexpr (!STATES) zv = E::one(r.z);
                if constexpr (STATES) steps += lanes.part == 0 ? sv : 0.0f;
                lds_s[slot][wave][lanes.channel * kTile + lanes.token] = sv;
                lds_u[slot][wave][lanes.channel * kTile + lanes.token] = sv * xv;
                r.b.store(lds_b[slot], p.N);
                if constexpr (!STATES) r.c.store(lds_c[slot], p.N);
                // (Now, or what is loaded next would go to other registers, and be moved when it is waited for.)
                asm volatile("" : "+v"(xv), "+v"(zv));
                __builtin_amdgcn_sched_barrier(0);
            };
            const auto finish = [&](int t, Buffer to, int tokens, float xv, float zv) {
                const float* q = lds_p[helper][wave] + product_at((lanes.channel * R + lanes.part) * 16) + lanes.token;
                float sum[4] = {};
#pragma unroll
                for (int n = 0; n < 16; ++n) sum[n % 4] += q[n * kPad];
                float out = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                if constexpr (R >= 4) out = swap_sum16(out, out);
                if constexpr (R >= 2) out = swap_sum32(out, out);
                out = fmaf(skip, xv, out);
                out = p.in.z ? out * (zv * sigmoid(zv)) : out;
                buffer_store<T>(E::to(t + tokens + lanes.token < at.live ? out : 0.0f), to,
                                at_y + (uint32_t)(tokens * (int)y.step));
            };
            if (tiles > 0) {
                // This helper's tiles are helper, helper + 2, ...; the step i of the states' waves is the tile i.
                const int own = at.first + helper * kTile;
                float xs[2], zs[2] = {};
                {
                    const Streams s = from(own), more = from(own + kRound * kTile);
                    fetch(raw[0], s, 0);
                    // (In this order, or the loop's first wait, for both ways into it, is for them all.)
                    __builtin_amdgcn_sched_barrier(0);
                    fetch(raw[1], s, 2 * kTile);
                    __builtin_amdgcn_sched_barrier(0);
                    prepare(raw[0], own, xs[0], zs[0], 0);
                    fetch(raw[0], more, 0);
                }
                __syncthreads();
                if (helper) __syncthreads();
                for (int i = 0; i < tiles; i += kRound) {
                    const int t = own + i * kTile;
                    const Streams s = from(t + (kRound + 2) * kTile);
                    const Buffer to = y.from(t);
                    // (Step i + helper: tile i + helper + 2 is made while it runs, its own outputs in the next.)
                    prepare(raw[1], t + 2 * kTile, xs[1], zs[1], 1);
                    fetch(raw[1], s, 0);
                    __syncthreads();
                    if constexpr (!STATES) finish(t, to, 0, xs[0], zs[0]);
                    __syncthreads();
                    prepare(raw[0], t + 4 * kTile, xs[0], zs[0], 0);
                    fetch(raw[0], s, 2 * kTile);
                    __syncthreads();
                    if constexpr (!STATES) finish(t, to, 2 * kTile, xs[1], zs[1]);
                    if (helper == 0 || i + kRound < tiles) __syncthreads();
                }
            }
            if constexpr (STATES) {
                // A channel's steps are in lanes CH apart.
#pragma unroll
                for (int m = Lanes<R>::CH; m < 64; m *= 2) steps += __shfl_xor(steps, m);
                lds_s[helper][wave][lane] = steps;   // (no longer needed for tiles)
            } else {
                for (int t = at.first + (tiles + helper) * kTile; t < at.end; t += 2 * kTile)
                    buffer_store<T>(E::to(0.0f), y.from(t), at_y);
            }
        } else {
            const bool state = FULL || at.n < p.N;
            float* carriers = p.carriers + (at.b * ((p.T + kTile - 1) / kTile) * p.D + at.row_d) * p.N + at.n;
            const float A = state ? finite(p.in.A[at.row_d * p.N + at.n] * kLog2e) : 0.0f;
            float h = 0.0f;
            if constexpr (!STATES) {
                if (state && p.chunks > 1) h = p.states[at.run(p)];
                else if (state && p.in.h0) h = p.in.h0[at.state(p)];
            }
            int buf = 0, block = at.first / kTile;
            const int row = lane / (16 * R) * kTile + lane % 16;
            const auto compute = [&](int out) {
                if constexpr (CARRY) {
                    if (state && block * kTile < at.end) carriers[block * (p.D * p.N)] = h;
                    ++block;
                }
                float b[kTile], c[kTile];
                const float s = lds_s[buf][wave][row], u = lds_u[buf][wave][row];
                read_tile(lds_b[buf] + at.n * kPad, b);
                if constexpr (!STATES) read_tile(lds_c[buf] + at.n * kPad, c);
                buf = (buf + 1) % kRound;
                each<kTile>([&](auto index) {
                    constexpr int tt = index;
                    h = fmaf(__builtin_amdgcn_exp2f(of_token<tt>(s) * A), h, of_token<tt>(u) * b[tt]);
                    if constexpr (!STATES) c[tt] = state ? c[tt] * h : 0.0f;
                });
                if constexpr (!STATES) {
                    float* q = lds_p[out][wave] + product_at(lane);
#pragma unroll
                    for (int k = 0; k < kTile; k += 4)
                        *(float4*)(q + k) = make_float4(c[k], c[k + 1], c[k + 2], c[k + 3]);
                }
            };
            if (tiles > 0) {
                __syncthreads();
                for (int i = 0; i < tiles; i += 2) {
                    compute(0);
                    __syncthreads();
                    compute(1);
                    __syncthreads();
                }
            }
            if constexpr (STATES) {
                if (state) p.states[at.run(p)] = h;
            } else {
                if (CARRY && state)
                    for (; block * kTile < at.end; ++block) carriers[block * (p.D * p.N)] = h;
                if (p.h_last && state && at.chunk == p.chunks - 1) p.h_last[at.state(p)] = h;
            }
        }
        __syncthreads();
        if constexpr (STATES) {
            if (helper == 0 && lane < Lanes<R>::CH)
                p.steps[(at.b * p.chunks + at.chunk) * p.D + at.d] = lds_s[0][wave][lane] + lds_s[1][wave][lane];
            __syncthreads();   // (the LDS has been read)
        }
    }
}

// h 2^e, where 2^e alone may leave float32 (a run's decays grow it past that and enter 0, or take what is large
// below it): the exponent's whole part goes into h's own.  |e| past 1024 makes 0 or infinity of any h, and 0 stays 0.
__device__ inline float scaled(float h, float e) {
    const float within = e > 1024.0f ? 1024.0f : e < -1024.0f ? -1024.0f : e, whole = __builtin_ceilf(within);
    return __builtin_ldexpf(h * __builtin_amdgcn_exp2f(within - whole), (int)whole);   // (a factor of 1/2 to 1; NaN stays NaN)
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
            h = scaled(h, rate * total) + own;
        }
        s[BACK ? 0 : (p.chunks - 1) * each] = h;
    }
}

// A few tokens: no tiles, nothing shared, a token after the other; the states move once.  Blocks are channels, groups
// and kTogether batches (divisions would cost as much as the rest), and no load is in a branch, so that all of them go
// ahead together: what is not there is read from where something else is, and left out.  128 requests of 4096 channels
// of 16 states take 17.4 us (21.7 with branches and divisions; one batch a thread 19.4, four 22.4).
//
// With LENGTHS a batch may have no token at all, and none of it is read then: its loads go to A (which has an element for
// each channel, and for each state).  Without, the lengths' absence is looked at all the same: known to the compiler, it
// orders the loads otherwise, and the 128 requests take 22.6 us; with the choice of A in both 19.2.
constexpr int kTogether = 2;
template <class E, int L, bool FULL, bool LENGTHS>
__global__ __launch_bounds__(64 * kWaves) void swr_scan_step_kernel(ScanParams p, int64_t first_tile) {
    typedef typename E::store T;
    constexpr int S = 4, M = kTogether;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n0 = lane % L * S;
    int64_t tile = first_tile + blockIdx.x;
    if (p.tiles % 8 == 0) tile = tile % 8 * (p.tiles / 8) + tile / 8;   // (as in Place)
    const int64_t c = (tile * kWaves + wave) * (64 / L) + lane / L;
    if (c >= p.Dg) return;
    int at[S];   // the states
    bool there[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        there[i] = FULL || n0 + i < p.N;
        at[i] = min(n0 + i, p.N - 1);
    }
    const auto states = [&](const float* row, float* h) {
        if constexpr (FULL) load_states<S, FULL>(row, n0, p.N, h);
        else {
#pragma unroll
            for (int i = 0; i < S; ++i) h[i] = row[at[i]];
        }
    };
    struct __attribute__((packed, aligned(sizeof(T)))) Four {
        T v[S];
    };
    const auto shared = [&](const T* row) {
        if constexpr (FULL) return *(const Four*)(row + n0);
        Four f;
#pragma unroll
        for (int i = 0; i < S; ++i) f.v[i] = row[at[i]];
        return f;
    };
    const bool has_z = p.in.z != nullptr, has_h = p.in.h0 != nullptr;
    for (int64_t group = blockIdx.y; group < p.G; group += gridDim.y) {
        const int64_t d = group * p.Dg + c;
        const float bias_there = (p.in.bias ? p.in.bias : p.in.A)[d], skip_there = (p.in.skip ? p.in.skip : p.in.A)[d];
        const float bias = p.in.bias ? bias_there : 0.0f, skip = p.in.skip ? skip_there : 0.0f;
        float A[S];
        states(p.in.A + d * p.N, A);
        for (int64_t b0 = (int64_t)blockIdx.z * M; b0 < p.B; b0 += (int64_t)gridDim.z * M) {
            float h[M][S];
            int64_t b[M], live[M];
#pragma unroll
            for (int m = 0; m < M; ++m) {   // (past the last batch that one once more)
                b[m] = min(b0 + m, p.B - 1);
                states((has_h ? p.in.h0 + (b[m] * p.D + d) * p.N : p.in.A + d * p.N), h[m]);
                live[m] = p.in.lengths ? min(max((int64_t)p.in.lengths[b[m]], (int64_t)0), p.T) : p.T;
            }
            for (int64_t t = 0; t < p.T; ++t) {
                T x[M], dt[M], z[M];
                Four bt[M], ct[M];
#pragma unroll
                for (int m = 0; m < M; ++m) {   // (past the batch's last token that one once more)
                    const int64_t tt = max(min(t, live[m] - 1), (int64_t)0);
                    const auto row = [&](const void* v, int64_t sb, int64_t s_t, int64_t more = 0) {
                        const T* at = (const T*)v + b[m] * sb + tt * s_t + more;
                        return !LENGTHS || live[m] > 0 ? at : (const T*)p.in.A;
                    };
                    x[m] = row(p.in.x, p.sx_b, p.sx_t)[d];
                    dt[m] = row(p.in.dt, p.sdt_b, p.sdt_t)[d];
                    z[m] = (has_z ? row(p.in.z, p.sz_b, p.sz_t) : row(p.in.x, p.sx_b, p.sx_t))[d];
                    bt[m] = shared(row(p.in.B, p.sB_b, p.sB_t, group * p.sB_g));
                    ct[m] = shared(row(p.in.C, p.sC_b, p.sC_t, group * p.sC_g));
                }
                if (t == 0) {
#pragma unroll
                    for (int i = 0; i < S; ++i) A[i] = finite(A[i] * (b0 == (int64_t)blockIdx.z * M ? kLog2e : 1.0f));
#pragma unroll
                    for (int m = 0; m < M; ++m) {
#pragma unroll
                        for (int i = 0; i < S; ++i) h[m][i] = has_h && there[i] ? h[m][i] : 0.0f;
                        if (p.carriers)   // (a single block of tokens)
                            store_states<S, FULL>(p.carriers + (b[m] * p.D + d) * p.N, n0, p.N, h[m]);
                    }
                }
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    const bool now = t < live[m];
                    const float xv = E::one(x[m]), zv = E::one(z[m]);
                    float s = E::one(dt[m]) + bias, v = 0.0f;
                    if (p.softplus) s = Softplus(s).value;
                    const float u = s * xv;
#pragma unroll
                    for (int i = 0; i < S; ++i) {
                        const float next = fmaf(__builtin_amdgcn_exp2f(s * A[i]), h[m][i], u * E::one(bt[m].v[i]));
                        h[m][i] = now && there[i] ? next : h[m][i];
                        v = there[i] ? fmaf(E::one(ct[m].v[i]), h[m][i], v) : v;
                    }
                    v = fmaf(skip, xv, lane_sum<L>(v));
                    if (has_z) v *= zv * sigmoid(zv);
                    if (lane % L == 0)
                        ((T*)p.y + b[m] * p.sy_b + t * p.sy_t)[d] = E::to(now ? v : 0.0f);
                }
            }
#pragma unroll
            for (int m = 0; m < M; ++m) {
                if (p.T == 0) {
#pragma unroll
                    for (int i = 0; i < S; ++i) h[m][i] = has_h && there[i] ? h[m][i] : 0.0f;
                }
                if (p.h_last) store_states<S, FULL>(p.h_last + (b[m] * p.D + d) * p.N, n0, p.N, h[m]);
            }
        }
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
                // (past the batch's last token 0 times its state, which may be infinite)
                if (tt < tokens && n < p.N) shares[tt * step + which * p.N + n] = t + tt < at.live ? sum : 0.0f;
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

// As swr_scan_back_states_kernel, a state a lane.
template <class E, int R, bool FULL>
__global__ __launch_bounds__(64 * kWaves) void swr_scan_back_rows_states_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int NP = 16 * R;
    __shared__ __attribute__((aligned(16))) float lds_c[2][NP * kPad];
    int buf = 0;
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const Place<NP> at(p, w);
        const int n = at.j, own = threadIdx.x % 16;
        const bool state = at.active && (FULL || n < p.N);
        const T* dt = (const T*)p.in.dt + at.b * p.sdt_b + at.d;
        const T* z = p.in.z ? (const T*)p.in.z + at.b * p.sz_b + at.d : nullptr;
        const T* dy = (const T*)p.dy + at.b * p.sy_b + at.d;
        const T* C = (const T*)p.in.C + at.b * p.sC_b + at.group * p.sC_g;
        const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
        const float A = state ? finite(p.in.A[(int64_t)at.d * p.N + n] * kLog2e) : 0.0f;
        float g = 0.0f, steps = 0.0f;
        T rdt = T(), rz = T(), rdy = T();
        SharedRows<E, NP, kWaves> rc;
        const auto fetch = [&](int64_t t) {
            if (t < at.first) return;
            const int64_t token = t + own;
            rdt = rz = rdy = T();
            if (at.active && token < at.live) {
                rdt = dt[token * p.sdt_t];
                if (z) rz = z[token * p.sz_t];
                rdy = dy[token * p.sy_t];
            }
            rc.load(C, p.sC_t, t, at.live - 1, p.N);
        };
        const int64_t last = at.first + (at.live - at.first + kTile - 1) / kTile * kTile - kTile;
        fetch(last);
        for (int64_t t = last; t >= at.first; t -= kTile, buf ^= 1) {
            const bool live = at.active && t + own < at.live;
            const float v = E::one(rdt) + bias, zv = E::one(rz);
            const float sv = !live ? 0.0f : p.softplus ? Softplus(v).value : v;
            const float wv = z ? E::one(rdy) * (zv * sigmoid(zv)) : E::one(rdy);
            steps += sv;
            rc.store(lds_c[buf], at.live - t, p.N);
            fetch(t - kTile);
            __syncthreads();
            float c[kTile];
            read_tile(lds_c[buf] + n * kPad, c);
            each<kTile>([&](auto index) {
                constexpr int tt = kTile - 1 - index;
                g = __builtin_amdgcn_exp2f(of_token<tt>(sv) * A) * fmaf(of_token<tt>(wv), c[tt], g);
            });
        }
        steps = lane_sum<16>(steps);
        if (state) p.states[at.states(p, at.chunk) + n] = g;
        if (at.active && n == 0) p.steps[(at.b * p.chunks + at.chunk) * p.D + at.d] = steps;
    }
}

// As swr_scan_back_kernel, a state a lane, the shares of dB and dC summed over a block of eight waves.
constexpr int kBackWaves = 8;
template <class E, int R, bool FULL>
__global__ __launch_bounds__(64 * kBackWaves) void swr_scan_back_rows_kernel(ScanParams p) {
    typedef typename E::store T;
    constexpr int NP = 16 * R;
    __shared__ __attribute__((aligned(16))) float lds_b[2][NP * kPad], lds_c[2][NP * kPad];
    __shared__ float lds_sum[kBackWaves][2][kTile][NP];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int buf = 0;
    for (int64_t w = blockIdx.x; w < p.work; w += gridDim.x) {
        const Place<NP, kBackWaves> at(p, w);
        const int n = at.j, own = threadIdx.x % 16;
        const bool state = at.active && (FULL || n < p.N);
        const T* x = (const T*)p.in.x + at.b * p.sx_b + at.d;
        const T* dt = (const T*)p.in.dt + at.b * p.sdt_b + at.d;
        const T* z = p.in.z ? (const T*)p.in.z + at.b * p.sz_b + at.d : nullptr;
        const T* dy = (const T*)p.dy + at.b * p.sy_b + at.d;
        const T* B = (const T*)p.in.B + at.b * p.sB_b + at.group * p.sB_g;
        const T* C = (const T*)p.in.C + at.b * p.sC_b + at.group * p.sC_g;
        const float bias = p.in.bias ? p.in.bias[at.d] : 0.0f;
        const float skip = p.in.skip ? p.in.skip[at.d] : 0.0f;
        const float A = state ? finite(p.in.A[(int64_t)at.d * p.N + n]) : 0.0f, A2 = finite(A * kLog2e);
        float g = 0.0f, dA = 0.0f, dbias = 0.0f, dskip = 0.0f;
        if (state && p.chunks > 1) g = p.states[at.states(p, at.chunk) + n];
        else if (state && p.dh_last) g = p.dh_last[(at.b * p.D + at.d) * p.N + n];
        T rx = T(), rdt = T(), rz = T(), rdy = T();
        float start = 0.0f;
        SharedRows<E, NP, kBackWaves> rb, rc;
        const auto fetch = [&](int64_t t) {
            if (t < at.first || t >= at.live) return;
            const int64_t token = t + own;
            rx = rdt = rz = rdy = T();
            if (at.active && token < at.live) {
                rx = x[token * p.sx_t];
                rdt = dt[token * p.sdt_t];
                if (z) rz = z[token * p.sz_t];
                rdy = dy[token * p.sy_t];
            }
            if (state)
                start = p.carriers_in[((at.b * ((p.T + kTile - 1) / kTile) + t / kTile) * p.D + at.d) * p.N + n];
            rb.load(B, p.sB_t, t, at.live - 1, p.N);
            rc.load(C, p.sC_t, t, at.live - 1, p.N);
        };
        const int64_t last = at.first + (at.end - at.first + kTile - 1) / kTile * kTile - kTile;
        fetch(last);
        for (int64_t t = last; t >= at.first; t -= kTile) {
            const int64_t tokens = min((int64_t)kTile, at.end - t);
            const int64_t out = (at.b * p.T + t + own) * p.D + at.d;
            const bool stores = at.active && n < 16 && own < tokens;
            float* shares = p.shares + (((at.b * p.T + t) * p.G + at.group) * p.tiles + at.tile) * 2 * p.N;
            const int64_t step = p.G * p.tiles * 2 * p.N;   // of the shares, from token to token
            if (t >= at.live) {   // past the batch's last token
                if (stores) {
                    ((T*)p.out.dx)[out] = ((T*)p.out.ddt)[out] = E::to(0.0f);
                    if (z) ((T*)p.out.dz)[out] = E::to(0.0f);
                }
                for (int e = threadIdx.x; e < kTile * 2 * NP; e += 64 * kBackWaves) {
                    const int tt = e / (2 * NP), which = e / NP % 2, m = e % NP;
                    if (tt < tokens && m < p.N) shares[tt * step + which * p.N + m] = 0.0f;
                }
                fetch(t - kTile);
                continue;
            }
            const bool live = at.active && t + own < at.live;
            const float v = E::one(rdt) + bias, xv = E::one(rx), zv = E::one(rz), dyv = E::one(rdy);
            float sv = v, slope = 1.0f;
            if (p.softplus) {
                const Softplus s(v);
                sv = s.value;
                slope = s.slope;
            }
            if (!live) sv = 0.0f;
            const float uv = sv * xv, gate = sigmoid(zv), wv = z ? dyv * (zv * gate) : dyv;
            float a[kTile], h[kTile + 1], b[kTile], c[kTile], f[kTile], q[kTile];
            h[0] = state ? start : 0.0f;
            rb.store(lds_b[buf], at.live - t, p.N);
            rc.store(lds_c[buf], at.live - t, p.N);
            fetch(t - kTile);
            __syncthreads();
            read_tile(lds_b[buf] + n * kPad, b);
            read_tile(lds_c[buf] + n * kPad, c);
            each<kTile>([&](auto index) {
                constexpr int tt = index;
                a[tt] = __builtin_amdgcn_exp2f(of_token<tt>(sv) * A2);
                h[tt + 1] = fmaf(a[tt], h[tt], of_token<tt>(uv) * b[tt]);
                f[tt] = c[tt] * h[tt + 1];
            });
            float yv = 0.0f;
            if (z) yv = state_sums<R>(f);
            each<kTile / 4>([&](auto index) {
                constexpr int first = kTile - 4 - 4 * index;
                float db[4], dc[4];
                each<4>([&](auto k) {
                    constexpr int tt = first + 3 - k;
                    const float wt = of_token<tt>(wv);
                    g = fmaf(wt, c[tt], g);
                    dc[3 - k] = wt * h[tt + 1];
                    db[3 - k] = of_token<tt>(uv) * g;
                    f[tt] = g * b[tt];
                    g *= a[tt];
                    const float past = g * h[tt];
                    q[tt] = past * A;
                    dA = fmaf(of_token<tt>(sv), past, dA);
                });
                // Sums over the wave's channels: of one channel (four rows) none, of two over halves.
                if constexpr (R == 1) {
                    const int tt = first + value_of_row(lane / 16);
                    lds_sum[wave][0][tt][n] = swap_sum16(swap_sum32(db[0], db[1]), swap_sum32(db[2], db[3]));
                    lds_sum[wave][1][tt][n] = swap_sum16(swap_sum32(dc[0], dc[1]), swap_sum32(dc[2], dc[3]));
                } else if constexpr (R == 2) {
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        lds_sum[wave][0][first + k + lane / 32][n] = swap_sum32(db[k], db[k + 1]);
                        lds_sum[wave][1][first + k + lane / 32][n] = swap_sum32(dc[k], dc[k + 1]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        lds_sum[wave][0][first + k][n] = db[k];
                        lds_sum[wave][1][first + k][n] = dc[k];
                    }
                }
            });
            const float along = state_sums<R>(f), decay = state_sums<R>(q);
            const float ddt = live ? fmaf(xv, along, decay) * slope : 0.0f;
            dbias += ddt;
            dskip = fmaf(wv, xv, dskip);
            if (stores) {
                ((T*)p.out.dx)[out] = E::to(live ? fmaf(sv, along, skip * wv) : 0.0f);
                ((T*)p.out.ddt)[out] = E::to(ddt);
                if (z)
                    ((T*)p.out.dz)[out] =
                        E::to(live ? dyv * fmaf(skip, xv, yv) * (gate * fmaf(zv, 1.0f - gate, 1.0f)) : 0.0f);
            }
            __syncthreads();
            for (int e = threadIdx.x; e < kTile * 2 * NP; e += 64 * kBackWaves) {
                const int tt = e / (2 * NP), which = e / NP % 2, m = e % NP;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < kBackWaves; ++i) sum += lds_sum[i][which][tt][m];
                if (tt < tokens && m < p.N) shares[tt * step + which * p.N + m] = t + tt < at.live ? sum : 0.0f;   // (as above)
            }
            buf ^= 1;
        }
        dbias = lane_sum<16>(dbias);
        dskip = lane_sum<16>(dskip);
        float* sums = p.sums + ((at.b * p.chunks + at.chunk) * p.D + at.d) * (p.N + 2);
        if (state) sums[n] = dA;
        if (at.active && n == 0) {
            sums[p.N] = dbias;
            sums[p.N + 1] = dskip;
        }
        if (p.out.dh0 && state && at.chunk == 0) p.out.dh0[(at.b * p.D + at.d) * p.N + n] = g;
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
constexpr int64_t kWant = 1024;   // waves: one for each of the GPU's SIMDs

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
hipError_t rows(const ScanPlan& plan, int N, F f) {
    const bool full = N == plan.lanes;
    switch (plan.lanes / 16) {
        case 1: return full ? f.template rows<1, true>() : f.template rows<1, false>();
        case 2: return full ? f.template rows<2, true>() : f.template rows<2, false>();
        case 4: return full ? f.template rows<4, true>() : f.template rows<4, false>();
    }
    return hipErrorInvalidValue;
}
template <class F>
hipError_t by_plan(const ScanPlan& plan, int N, const F& f) {
    return plan.states == 1 ? rows(plan, N, f) : narrow(plan, N, f);
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
    template <int R, bool FULL>
    hipError_t rows() const {
        if (!STATES && p.carriers)
            hipLaunchKernelGGL((swr_scan_rows_kernel<E, R, FULL, false, true>), dim3(grid_of(p.work)), dim3(192 * kWaves),
                               0, st, p);
        else
            hipLaunchKernelGGL((swr_scan_rows_kernel<E, R, FULL, STATES, false>), dim3(grid_of(p.work)),
                               dim3(192 * kWaves), 0, st, p);
        return hipGetLastError();
    }
};
template <class E>
struct Step {
    const ScanParams& p;
    hipStream_t st;
    template <int L, int S, bool FULL>
    hipError_t operator()() const {
        const auto kernel = p.in.lengths ? swr_scan_step_kernel<E, L, FULL, true> : swr_scan_step_kernel<E, L, FULL, false>;
        // (A launch has less than 2^32 threads along a dimension.)
        constexpr int64_t kMostTiles = (int64_t)1 << 23;
        for (int64_t first = 0; first < p.tiles; first += kMostTiles) {
            const dim3 grid((unsigned)std::min(p.tiles - first, kMostTiles), (unsigned)std::min<int64_t>(p.G, 65535),
                            (unsigned)std::min<int64_t>((p.B + kTogether - 1) / kTogether, 65535));
            hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), 0, st, p, first);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
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
    template <int R, bool FULL>
    hipError_t rows() const {   // (blocks of half as many waves as those of the last pass: twice as many)
        ScanParams q = p;
        q.tiles = (p.Dg + kWaves * 4 / R - 1) / (kWaves * 4 / R);
        q.work = p.B * p.G * q.tiles * p.chunks;
        hipLaunchKernelGGL((swr_scan_back_rows_states_kernel<E, R, FULL>), dim3(grid_of(q.work)), dim3(64 * kWaves), 0, st,
                           q);
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
    template <int R, bool FULL>
    hipError_t rows() const {
        hipLaunchKernelGGL((swr_scan_back_rows_kernel<E, R, FULL>), dim3(grid_of(p.work)), dim3(64 * kBackWaves), 0, st,
                           p);
        return hipGetLastError();
    }
};

template <class E>
hipError_t forward(const ScanPlan& plan, const ScanParams& p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (p.T <= kFew) return narrow(plan, p.N, Step<E>{p, st});
    if (plan.chunks > 1) {
        const Forward<E, true> states{p, st};
        if ((e = by_plan(plan, p.N, states)) != hipSuccess) return e;
        hipLaunchKernelGGL(swr_scan_chain_kernel<false>, dim3(grid_of((p.B * p.D * p.N + 255) / 256)), dim3(256), 0, st,
                           p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const Forward<E, false> all{p, st};
    return by_plan(plan, p.N, all);
}

template <class E>
hipError_t backward(const ScanPlan& plan, const ScanParams& p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (plan.chunks > 1) {
        const BackStates<E> states{p, st};
        if ((e = plan.states == 1 ? rows(plan, p.N, states) : narrow(plan, p.N, states)) != hipSuccess) return e;
        hipLaunchKernelGGL(swr_scan_chain_kernel<true>, dim3(grid_of((p.B * p.D * p.N + 255) / 256)), dim3(256), 0, st,
                           p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const Back<E> back{p, st};
    if ((e = plan.states == 1 ? rows(plan, p.N, back) : narrow(plan, p.N, back)) != hipSuccess) return e;
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
    const int64_t dg = p.D / p.G;
    const auto make = [&](int states) {
        ScanPlan plan = {};
        plan.states = states;
        plan.lanes = states == 1 ? (p.N <= 16 ? 16 : p.N <= 32 ? 32 : 64) : lanes_of(p.N, states);
        const int64_t channels = (states == 1 && backward ? kBackWaves : kWaves) * (64 / plan.lanes);
        plan.tiles = (dg + channels - 1) / channels;
        plan.chunks = 1;
        plan.chunk = std::max<int64_t>(kTile, (p.T + kTile - 1) / kTile * kTile);
        return plan;
    };
    if (p.T <= kFew && !backward) return make(4);
    // (48 tokens have to lie within 31 bits of bytes where a lane has a state.)
    bool near = p.D <= 1 << 26;
    for (const int64_t s : {p.sx_t, p.sdt_t, p.sz_t, p.sy_t, p.sB_t, p.sC_t}) near = near && s <= 1 << 22;
    ScanPlan plan = make(p.N > 8 && near ? 1 : 4);
    const int64_t waves = plan.states == 1 && backward ? kBackWaves : kWaves;
    // Runs of at least 64 tokens, as many as give every SIMD a wave.  8192 tokens of 16 states cut and whole: of 1024
    // channels 113 and 240 us forward, 487 and 1460 backward; of 2048 208 and 241, 957 and 1443; of 2560 to 3584, in two runs,
    // 300 and 242, 1032 and 1530 (a forward there would be faster whole); of 4 states and 2048 channels 171 and 3017, 272 and 5322.
    const int64_t one = std::max<int64_t>(1, plan.blocks(p.B, p.G) * waves);   // (a batch of none has none)
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
