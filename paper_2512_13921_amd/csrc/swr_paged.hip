// swr_paged.hip -- the paged key-value cache on gfx950: tables and slot maps
// from the requests' lengths, new keys and values into their slots, and the
// attention of one query token a request over its cached tokens.
#include <algorithm>

#include "swr_hybrid_launch.h"

namespace swr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------
// Tables
// ---------------------------------------------------------------------------

// Inclusive sums of a and b over the block's 256 threads.
__device__ inline void block_scan(int64_t& a, int64_t& b, int64_t (*buf)[2]) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int64_t pa = __shfl_up(a, m), pb = __shfl_up(b, m);
        if (lane >= m) { a += pa; b += pb; }
    }
    __syncthreads();   // (the last chunk's sums have been read)
    if (lane == 63) { buf[wave][0] = a; buf[wave][1] = b; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 3; ++w)
        if (w < wave) { a += buf[w][0]; b += buf[w][1]; }
}

constexpr int kTableTokens = 1024;   // slots a block writes

// The last of 256 entries whose first (ascending; entry 0's is at most t) is at most t.
__device__ inline int holder(const int64_t* first, int64_t t) {
    int r = 0;
#pragma unroll
    for (int step = 128; step > 0; step >>= 1)
        if (first[r + step] <= t) r += step;
    return r;
}

// Every block sums the requests' new tokens and pages itself, 256 requests at
// a time (sums of a launch before it would cost that launch, and the lengths are
// a few KB in the L2), and writes its range of the slots and every
// gridDim.x-th 256 of the new pages' entries.  The entries that it reads, of pages
// that a request held before, are none that a block writes.
__global__ __launch_bounds__(256) void swr_tables_kernel(TableParams p) {
    __shared__ int64_t buf[4][2];
    __shared__ int64_t first_token[257], first_page[257];
    __shared__ int32_t length[256];
    const int64_t lo = (int64_t)blockIdx.x * kTableTokens, hi = min(lo + kTableTokens, p.tokens);
    const int64_t count = min(max(p.count[0], 0), p.free_pages);
    int64_t tokens = 0, pages = 0;   // new ones of the requests before this chunk
    for (int c = 0; c < p.batch; c += 256) {
        const int i = c + (int)threadIdx.x;
        const int64_t len = i < p.batch ? max(p.lengths[i], 0) : 0, more = i < p.batch ? max(p.news[i], 0) : 0;
        const int64_t held = (len + p.page_size - 1) / p.page_size;
        const int64_t after = (len + more + p.page_size - 1) / p.page_size;
        const int64_t need = max(min(after, (int64_t)p.max_pages) - held, (int64_t)0);
        int64_t ta = more, pa = need;
        block_scan(ta, pa, buf);   // (its barriers stand between the last chunk's readers and these writes)
        ta += tokens;
        pa += pages;
        first_token[threadIdx.x] = ta - more;
        first_page[threadIdx.x] = pa - need;
        length[threadIdx.x] = (int32_t)len;
        if (threadIdx.x == 255) { first_token[256] = ta; first_page[256] = pa; }
        __syncthreads();
        if (blockIdx.x == 0 && i < p.batch) {
            p.starts[i] = (int32_t)min(ta - more, (int64_t)0x7fffffff);
            p.new_lengths[i] = (int32_t)min(len + more, (int64_t)0x7fffffff);
        }
        // New pages' entries.
        for (int64_t k = pages + (int64_t)blockIdx.x * 256 + threadIdx.x; k < first_page[256];
             k += (int64_t)gridDim.x * 256) {
            const int r = holder(first_page, k);
            const int64_t old = ((int64_t)length[r] + p.page_size - 1) / p.page_size;
            p.table[(c + r) * p.st + old + (k - first_page[r])] = k < count ? p.stack[count - 1 - k] : -1;
        }
        // Slots of this block's tokens that are this chunk's requests'.
        for (int64_t t = max(lo, tokens) + threadIdx.x; t < min(hi, first_token[256]); t += 256) {
            const int r = holder(first_token, t);
            const int64_t at = length[r] + (t - first_token[r]), page = at / p.page_size;
            const int64_t old = ((int64_t)length[r] + p.page_size - 1) / p.page_size;
            const int64_t k = first_page[r] + (page - old);
            int64_t id = -1;
            if (page < p.max_pages)
                id = page < old ? p.table[(c + r) * p.st + page] : k < count ? p.stack[count - 1 - k] : -1;
            p.slots[t] = id >= 0 ? id * p.page_size + at % p.page_size : -1;
        }
        tokens = first_token[256];
        pages = first_page[256];
    }
    for (int64_t t = max(lo, tokens) + threadIdx.x; t < hi; t += 256) p.slots[t] = -1;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.starts[p.batch] = (int32_t)min(tokens, (int64_t)0x7fffffff);
        p.new_count[0] = (int32_t)max(count - pages, (int64_t)0);
    }
}

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

// A copy of 16-byte vectors; keys in the grid's first half of y, values in the second.
__global__ __launch_bounds__(256) void swr_append_kernel(AppendParams p) {
    const bool values = blockIdx.y != 0;
    const u32x4* in = (const u32x4*)(values ? p.v : p.k);
    u32x4* out = (u32x4*)(values ? p.v_cache : p.k_cache);
    const int64_t st = values ? p.sv_t : p.sk_t, sh = values ? p.sv_h : p.sk_h;
    const int64_t total = p.tokens * p.per_token;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / p.per_token;
        const uint32_t e = (uint32_t)(i - t * p.per_token), head = e / p.per_head, c = e - head * p.per_head;
        const int64_t slot = p.slots[t];
        if (slot < 0 || slot >= p.rows) continue;
        const int64_t page = slot / p.page_size, at = slot - page * p.page_size;
        out[page * p.s_page + at * p.s_token + head * p.s_head + c] = in[t * st + head * sh + c];
    }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
//
// The query heads that share a key head (up to 16; more are further "head
// tiles") are the columns of 16 x 16 matrix products, cached tokens their rows:
//     S[t, g] = K[t, :] . q[g, :]        then        Y[c, g] += sum_t V[t, c] P[t, g]
// A wave takes 32 tokens at a time.  Lane (l = lane % 16, quarter u = lane / 16)
// holds column g = l of S at tokens 16 s + 4 u + i (s < 2, i < 4), which is where
// the second product wants P: the order of its contraction index is free, so V's rows
// are loaded for those tokens, and no lane exchanges P with another.  K and V go
// from memory to registers, with no LDS between.  P is split into two
// bf16 parts (float32 caches use float32 products throughout), so that y is
// rounded once.  Maxima and sums are float32; a lane's sums are joined at the end.
//
// The work, (request, key head) rows of ceil(tokens / 32) tiles, is laid end to
// end and cut into equal shares, one a workgroup: every workgroup finds its own share
// from the lengths, so a long request among short ones costs no idle
// workgroups, and no host knows the lengths.  Waves take a row's tiles in turn
// and are joined in LDS.  A row cut between workgroups leaves its
// parts in the workspace, which swr_paged_join_kernel joins.

constexpr int kTile = 32;      // tokens of a wave's tile
constexpr int kWaves = 4;
constexpr uint32_t kNoRow = 0xffffffffu;

// Tiles and first position of request b.
struct Rows {
    int64_t low;
    int tiles, length;
};
__device__ inline Rows rows_of(const PagedParams& p, int b) {
    const int64_t most = (int64_t)p.max_pages * p.page_size;
    const int64_t n = max(p.lengths[b], 0), low = p.window > 0 ? max(n - p.window, (int64_t)0) : 0;
    const int64_t end = min(n, most);   // (positions past the table are left out)
    return {low, end > low ? (int)((end - low + kTile - 1) / kTile) : 0, (int)end};
}

// Where the flat order of tiles stands: (request, head row within the request,
// tile within the row), and the share of each workgroup.
struct Place {
    int64_t total;   // tiles of all rows
    int64_t per;     // tiles a workgroup
    int b;           // the request that holds tile `at`, and the tiles before it
    int64_t before;
};

// The place of flat tile `at(per)`, found by the whole block; buf holds 6 values.
template <class At>
__device__ inline Place find(const PagedParams& p, int heads, int64_t* buf, At at) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t sum = 0;
    for (int b = threadIdx.x; b < p.batch; b += 256) sum += rows_of(p, b).tiles;
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) buf[wave] = sum;
    __syncthreads();
    Place f;
    f.total = (buf[0] + buf[1] + buf[2] + buf[3]) * heads;
    f.per = max((f.total + p.workgroups - 1) / p.workgroups, (int64_t)kWaves);
    const int64_t want = at(f.per);
    int64_t before = 0;
    f.b = p.batch;
    f.before = f.total;
    for (int c = 0; c < p.batch && want < f.total; c += 256) {
        const int b = c + (int)threadIdx.x;
        const int64_t n = b < p.batch ? (int64_t)rows_of(p, b).tiles * heads : 0;
        int64_t s = n;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int64_t u = __shfl_up(s, m);
            if (lane >= m) s += u;
        }
        __syncthreads();
        if (lane == 63) buf[wave] = s;
        __syncthreads();
        for (int w = 0; w < wave; ++w) s += buf[w];
        s += before;
        if (s > want && s - n <= want) { buf[4] = b; buf[5] = s - n; }
        before += buf[0] + buf[1] + buf[2] + buf[3];
        if (before > want) break;   // (uniform)
    }
    __syncthreads();
    if (want < f.total) { f.b = (int)buf[4]; f.before = buf[5]; }
    return f;
}

struct B16 {
    typedef uint16_t T;
};
struct B32 {
    typedef float T;
};

__device__ inline float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }

// A column's running maximum (the same on its four lanes) and this lane's sum
// of the weights against it.
struct Running {
    float m = -INFINITY, sum = 0.0f;

    // Scores (times log2 e) to weights against the running maximum; returns
    // what the sums so far are multiplied by.
    __device__ float weigh(float (&p)[8]) {
        float top = m;
#pragma unroll
        for (int t = 0; t < 8; ++t) top = fmaxf(top, p[t]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.0f : top;   // (nothing yet: weights of 0, not NaN)
        const float alpha = exp2f(m - base);
        m = top;
        float s = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            p[t] = exp2f(p[t] - base);
            s += p[t];
        }
        sum = sum * alpha + s;
        return alpha;
    }
};

// One wave's state of one row: columns g = l.
template <class E, int DP>
struct State;

// bf16: DP = 32, 64, 128 or 256 channels (D rounded up).  Lane (l, u) holds
// channels 32 c + 8 u .. + 7 of K's token row l, and channels l * CH .. of V's rows.
template <int DP>
struct State<B16, DP> {
    static constexpr int CH = DP / 16;          // channels of V that a lane holds
    static constexpr int NK = DP / 32;
    bf16x8 q[NK];
    f32x4 acc[CH];                              // acc[j]: channels (4 u + i) * CH + j, column l
    Running run;

    __device__ void begin(const uint16_t* qrow, bool in, int u, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            u32x4 v{0, 0, 0, 0};
            if (in && 32 * c + 8 * u < D) v = *(const u32x4*)(qrow + 32 * c + 8 * u);
            q[c] = __builtin_bit_cast(bf16x8, v);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) acc[j] = f32x4{0, 0, 0, 0};
    }

    // 32 tokens: lane i < 32 has token i's row (16-byte units, kNoRow: none).
    __device__ void tile(const u32x4* kb, const u32x4* vb, uint32_t row, int l, int u, int D, float scale) {
        u32x4 k[2][NK];
        uint32_t v[8][CH / 2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t r = (uint32_t)__shfl((int)row, 16 * s + l);
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                k[s][c] = u32x4{0, 0, 0, 0};
                if (r != kNoRow && 32 * c + 8 * u < D) k[s][c] = kb[(int64_t)r + 4 * c + u];
            }
        }
        bool in[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t r = (uint32_t)__shfl((int)row, 16 * (t / 4) + 4 * u + t % 4);
            in[t] = r != kNoRow;
            const bool ok = in[t] && l * CH < D;
            const uint32_t* at = (const uint32_t*)(vb + (int64_t)(in[t] ? r : 0)) + l * (CH / 2);
            if constexpr (CH == 2) {
                v[t][0] = ok ? *at : 0;
            } else if constexpr (CH == 4) {
                const u32x2 w = ok ? *(const u32x2*)at : u32x2{0, 0};
                v[t][0] = w[0]; v[t][1] = w[1];
            } else {
#pragma unroll
                for (int h = 0; h < CH / 8; ++h) {
                    const u32x4 w = ok ? *(const u32x4*)(at + 4 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[t][4 * h + i] = w[i];
                }
            }
        }
        float p[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f32x4 x{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NK; ++c)
                x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[s][c]), q[c], x, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * s + i] = in[4 * s + i] ? x[i] * scale : -INFINITY;
        }
        const float alpha = run.weigh(p);
        bf16x8 hi, lo;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            hi[t] = (__bf16)p[t];
            lo[t] = (__bf16)(p[t] - (float)hi[t]);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            // Channel l * CH + j of the lane's 8 tokens.
            u32x4 a;
#pragma unroll
            for (int t = 0; t < 4; ++t)
                a[t] = __builtin_amdgcn_perm(v[2 * t + 1][j / 2], v[2 * t][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            const bf16x8 w = __builtin_bit_cast(bf16x8, a);
            f32x4 y = acc[j] * alpha;
            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, hi, y, 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, lo, y, 0, 0, 0);
        }
    }
};

// float32: lane (l, u) holds channels 16 c + 4 u .. + 3 of K's token row l.
template <int DP>
struct State<B32, DP> {
    static constexpr int CH = DP / 16;
    static constexpr int NK = DP / 16;
    f32x4 q[NK];
    f32x4 acc[CH];
    Running run;

    __device__ void begin(const float* qrow, bool in, int u, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            q[c] = f32x4{0, 0, 0, 0};
            if (in && 16 * c + 4 * u < D) q[c] = *(const f32x4*)(qrow + 16 * c + 4 * u);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) acc[j] = f32x4{0, 0, 0, 0};
    }

    __device__ void tile(const u32x4* kb, const u32x4* vb, uint32_t row, int l, int u, int D, float scale) {
        float p[8];
        bool in[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t r = (uint32_t)__shfl((int)row, 16 * s + l);
            f32x4 x{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                u32x4 k{0, 0, 0, 0};
                if (r != kNoRow && 16 * c + 4 * u < D) k = kb[(int64_t)r + 4 * c + u];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x = __builtin_amdgcn_mfma_f32_16x16x4f32(as_float(k[i]), q[c][i], x, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                in[4 * s + i] = (uint32_t)__shfl((int)row, 16 * s + 4 * u + i) != kNoRow;
                p[4 * s + i] = in[4 * s + i] ? x[i] * scale : -INFINITY;
            }
        }
        const float alpha = run.weigh(p);
#pragma unroll
        for (int j = 0; j < CH; ++j) acc[j] *= alpha;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t r = (uint32_t)__shfl((int)row, 16 * (t / 4) + 4 * u + t % 4);
            const float* at = (const float*)(vb + (int64_t)(in[t] ? r : 0)) + l * CH;
            float v[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] = in[t] && l * CH < D ? at[j] : 0.0f;
#pragma unroll
            for (int j = 0; j < CH; ++j)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], p[t], acc[j], 0, 0, 0);
        }
    }
};

__device__ inline void put(uint16_t* y, float f) { *y = __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ inline void put(float* y, float f) { *y = f; }

constexpr float kLn2 = 0.69314718055994530942f;

// Channel c of a row's output from its weighted sum and the weights' sum, which
// is 0 where the row has no token (a token of the maximum weighs 1).
template <class T>
__device__ inline void finish(const PagedParams& p, int b, int64_t head, int c, float m, float y, float sum) {
    if (c < p.D) put((T*)p.y + b * p.sy_b + head * p.sy_h + c, sum == 0.0f ? 0.0f : y / sum);
    if (c == 0 && p.lse)
        p.lse[(int64_t)b * p.kv_heads * p.group + head] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * kLn2;
}

// Floats of a row part in the workspace: 16 columns of DP channels, maxima, sums.
constexpr int64_t part_floats(int dp) { return 16 * ((int64_t)dp + 2); }

template <class E, int DP>
__global__ __launch_bounds__(kWaves * 64) void swr_paged_kernel(PagedParams p) {
    typedef typename E::T T;
    typedef State<E, DP> S;
    constexpr int CH = S::CH;
    __shared__ int64_t buf[6];
    __shared__ float join_m[kWaves][16], join_s[kWaves][16];
    __shared__ float join[kWaves][DP][17];   // (17: the lanes' columns fall on different banks)
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 16, u = lane / 16;
    const int heads = p.kv_heads * p.head_tiles;
    const Place f = find(p, heads, buf, [&](int64_t per) { return blockIdx.x * per; });
    int64_t at = blockIdx.x * f.per;
    const int64_t end = min(at + f.per, f.total);
    int64_t before = f.before;
    for (int b = f.b; at < end; ++b) {
        const Rows r = rows_of(p, b);
        if (r.tiles == 0) continue;
        for (int64_t h = (at - before) / r.tiles; h < heads && at < end; ++h) {
            const int64_t row0 = before + h * r.tiles;   // the row's tiles: row0 .. row0 + r.tiles
            const int t0 = (int)(at - row0), t1 = (int)min((int64_t)r.tiles, end - row0);
            const int kv = (int)(h / p.head_tiles), g0 = (int)(h % p.head_tiles) * 16;
            const int columns = min(p.group - g0, 16);
            const int64_t head = (int64_t)kv * p.group + g0;
            S s;
            s.begin((const T*)p.q + b * p.sq_b + (head + min(l, columns - 1)) * p.sq_h, l < columns, u, p.D);
            const u32x4* kb = (const u32x4*)p.k + (int64_t)kv * p.s_head;
            const u32x4* vb = (const u32x4*)p.v + (int64_t)kv * p.s_head;
            for (int t = t0 + wave; t < t1; t += kWaves) {
                const int64_t pos = r.low + (int64_t)t * kTile + lane % kTile;
                uint32_t row = kNoRow;
                if (pos < r.length) {
                    const uint32_t page = (uint32_t)pos / (uint32_t)p.page_size;
                    const int id = p.table[b * p.st + page];
                    if (id >= 0 && id < p.pages)
                        row = (uint32_t)id * p.s_page + ((uint32_t)pos - page * p.page_size) * p.s_token;
                }
                s.tile(kb, vb, row, l, u, p.D, p.scale_log2);
            }
            // The waves' parts, joined.
            s.run.sum += __shfl_xor(s.run.sum, 16);
            s.run.sum += __shfl_xor(s.run.sum, 32);
            __syncthreads();   // (the last row's parts have been read)
            if (u == 0) { join_m[wave][l] = s.run.m; join_s[wave][l] = s.run.sum; }
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) join[wave][(4 * u + i) * CH + j][l] = s.acc[j][i];
            __syncthreads();
            const bool whole = t0 == 0 && t1 == r.tiles;
            float* part = p.part + (blockIdx.x * 2 + (t0 == 0 && at > blockIdx.x * f.per ? 1 : 0)) * part_floats(DP);
            for (int e = threadIdx.x; e < columns * DP; e += kWaves * 64) {
                const int g = e / DP, c = e % DP;
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) m = fmaxf(m, join_m[w][g]);
                const float base = m == -INFINITY ? 0.0f : m;
                float y = 0.0f, sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float a = exp2f(join_m[w][g] - base);
                    y += join[w][c][g] * a;
                    sum += join_s[w][g] * a;
                }
                if (whole) {
                    finish<T>(p, b, head + g, c, m, y, sum);
                } else {
                    part[g * (DP + 2) + c] = y;
                    if (c == 0) { part[g * (DP + 2) + DP] = m; part[g * (DP + 2) + DP + 1] = sum; }
                }
            }
            at = row0 + t1;
        }
        before += (int64_t)r.tiles * heads;
    }
}

// Rows that were cut between workgroups: their parts, in order.  Rows without
// tokens: zeros.  A block takes a row (request, key head, head tile).
template <class E, int DP>
__global__ __launch_bounds__(256) void swr_paged_join_kernel(PagedParams p) {
    typedef typename E::T T;
    __shared__ int64_t buf[8];
    const int heads = p.kv_heads * p.head_tiles;
    const int b = (int)(blockIdx.x / heads), h = (int)(blockIdx.x % heads);
    // Tiles of all requests, and of those before b.
    int64_t all = 0, prior = 0;
    for (int i = threadIdx.x; i < p.batch; i += 256) {
        const int n = rows_of(p, i).tiles;
        all += n;
        if (i < b) prior += n;
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
        all += __shfl_xor(all, m);
        prior += __shfl_xor(prior, m);
    }
    if (threadIdx.x % 64 == 0) { buf[threadIdx.x / 64 * 2] = all; buf[threadIdx.x / 64 * 2 + 1] = prior; }
    __syncthreads();
    const int64_t total = (buf[0] + buf[2] + buf[4] + buf[6]) * heads;
    const int64_t per = max((total + p.workgroups - 1) / p.workgroups, (int64_t)kWaves);
    const Rows r = rows_of(p, b);
    const int64_t row0 = (buf[1] + buf[3] + buf[5] + buf[7]) * heads + (int64_t)h * r.tiles;
    const int64_t w0 = row0 / per, w1 = r.tiles ? (row0 + r.tiles - 1) / per : w0 - 1;
    if (w0 == w1) return;
    const int kv = h / p.head_tiles, g0 = h % p.head_tiles * 16, columns = min(p.group - g0, 16);
    const int64_t head = (int64_t)kv * p.group + g0;
    // The first part is the first of its workgroup if the row starts that workgroup's share.
    const int64_t first = w0 * 2 + (row0 > w0 * per ? 1 : 0);
    for (int e = threadIdx.x; e < columns * DP; e += 256) {
        const int g = e / DP, c = e % DP;
        float m = -INFINITY, y = 0.0f, sum = 0.0f;
        for (int64_t w = w0; w <= w1; ++w) {
            const float* part = p.part + (w == w0 ? first : 2 * w) * part_floats(DP) + g * (DP + 2);
            const float pm = part[DP], top = fmaxf(m, pm), base = top == -INFINITY ? 0.0f : top;
            const float a = exp2f(m - base), z = exp2f(pm - base);
            y = y * a + part[c] * z;
            sum = sum * a + part[DP + 1] * z;
            m = top;
        }
        finish<T>(p, b, head + g, c, m, y, sum);
    }
}

int padded(int64_t D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256; }

template <class E, int DP>
hipError_t go(const PagedParams& p, hipStream_t st) {
    hipLaunchKernelGGL((swr_paged_kernel<E, DP>), dim3((unsigned)p.workgroups), dim3(kWaves * 64), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((swr_paged_join_kernel<E, DP>), dim3((unsigned)(p.batch * p.kv_heads * p.head_tiles)), dim3(256),
                       0, st, p);
    return hipGetLastError();
}

template <class E>
hipError_t by_width(const PagedParams& p, hipStream_t st) {
    switch (padded(p.D)) {
        case 32: return go<E, 32>(p, st);
        case 64: return go<E, 64>(p, st);
        case 128: return go<E, 128>(p, st);
        default: return go<E, 256>(p, st);
    }
}

}  // namespace

int paged_workgroups(const swr_paged_t& p) {
    const int64_t positions = p.window > 0 ? std::min(p.window, p.max_pages * p.cache.page_size)
                                           : p.max_pages * p.cache.page_size;
    const int64_t heads = p.cache.heads * ((p.q_heads / p.cache.heads + 15) / 16);
    const double tiles = (double)p.batch * (double)heads * (double)((positions + kTile - 1) / kTile);
    return (int)std::max(1.0, std::min(1024.0, (tiles + kWaves - 1) / kWaves));
}

int64_t paged_part_floats(const swr_paged_t& p) { return part_floats(padded(p.cache.D)); }

hipError_t launch_tables(const TableParams& p, void* stream) {
    const int64_t blocks = std::max<int64_t>(1, (p.tokens + kTableTokens - 1) / kTableTokens);
    hipLaunchKernelGGL(swr_tables_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, p);
    return hipGetLastError();
}

hipError_t launch_append(const AppendParams& p, void* stream) {
    const int64_t blocks = std::min<int64_t>((p.tokens * p.per_token + 255) / 256, 8192);
    hipLaunchKernelGGL(swr_append_kernel, dim3((unsigned)blocks, 2), dim3(256), 0, (hipStream_t)stream, p);
    return hipGetLastError();
}

hipError_t launch_paged(int dtype, const PagedParams& p, void* stream) {
    return dtype == SWR_DTYPE_BF16 ? by_width<B16>(p, (hipStream_t)stream) : by_width<B32>(p, (hipStream_t)stream);
}

}  // namespace swr
