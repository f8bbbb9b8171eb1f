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

// Slots a block writes.  (1024: 6.2 us where 1000 new tokens of one request take 3.7, 6.6 for
// 6.1 at 200 x 1311.)
constexpr int kTableTokens = 256;

// The last of 256 entries whose first (ascending; entry 0's is at most t) is at most t.
__device__ inline int holder(const int64_t* first, int64_t t) {
    int r = 0;
#pragma unroll
    for (int step = 128; step > 0; step >>= 1)
        if (first[r + step] <= t) r += step;
    return r;
}

// n / page_size; a division of 64 bits (about 100 instructions) past 2^31 only.
__device__ inline int64_t over(const TableParams& p, int64_t n) {
    return n < (int64_t)1 << 31 ? (int64_t)p.page.over((uint32_t)n) : n / p.page_size;
}

// Every block sums the requests' new tokens and pages itself, 256 requests at
// a time (sums of a launch before it would cost that launch, and the lengths are
// a few KB in the L2; 8 requests of one token 3.1 us, 200 of 1311 6.0, all of it
// the chain of lengths, sums, search, page and slot), and writes its range of the slots and every
// gridDim.x-th 256 of the new pages' entries.  The entries that it reads, of pages
// that a request held before, are none that a block writes.
__global__ __launch_bounds__(256) void swr_tables_kernel(TableParams p) {
    __shared__ int64_t buf[4][2];
    __shared__ int64_t first_token[257], first_page[257];
    __shared__ int32_t length[256];
    const int64_t lo = (int64_t)blockIdx.x * kTableTokens, hi = min(lo + kTableTokens, p.tokens);
    const int64_t count = min(max(p.count[0], 0), p.free_pages);
    int64_t tokens = 0, pages = 0;   // new ones of the requests before this chunk
    int i = threadIdx.x;
    int next_len = i < p.batch ? p.lengths[i] : 0, next_more = i < p.batch ? p.news[i] : 0;
    for (int c = 0; c < p.batch; c += 256, i += 256) {
        const int64_t len = max(next_len, 0), more = max(next_more, 0);
        if (c + 256 < p.batch) {   // the next chunk's, on their way while this one is worked on
            next_len = i + 256 < p.batch ? p.lengths[i + 256] : 0;
            next_more = i + 256 < p.batch ? p.news[i + 256] : 0;
        }
        const int64_t held = over(p, len + p.page_size - 1), after = over(p, len + more + p.page_size - 1);
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
            const int64_t old = over(p, (int64_t)length[r] + p.page_size - 1);
            p.table[(c + r) * p.st + old + (k - first_page[r])] = k < count ? p.stack[count - 1 - k] : -1;
        }
        // Slots of this block's tokens that are this chunk's requests'.
        for (int64_t t = max(lo, tokens) + threadIdx.x; t < min(hi, first_token[256]); t += 256) {
            const int r = holder(first_token, t);
            const int64_t at = length[r] + (t - first_token[r]), page = over(p, at);
            const int64_t old = over(p, (int64_t)length[r] + p.page_size - 1);
            const int64_t k = first_page[r] + (page - old);
            int64_t id = -1;
            if (page < p.max_pages)
                id = page < old ? p.table[(c + r) * p.st + page] : k < count ? p.stack[count - 1 - k] : -1;
            p.slots[t] = id >= 0 ? id * p.page_size + (at - page * p.page_size) : -1;
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

// Bound by its bytes: 50021 tokens of 8 heads of 128, bf16, 73 us, 5.6 TB/s; 256
// tokens 2.9 us, a launch.  A copy of 16-byte vectors; keys in the grid's first half of y, values in the second.
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
// from memory to registers, with no LDS between.  Against bf16 values P is cut into three
// bf16 parts, all 24 of its bits (float32 caches use float32 products throughout), so that y is
// rounded once.  Maxima and sums are float32; a lane's sums are joined at the end.
//
// The work, (request, key head) rows of ceil(tokens / 32) tiles, is laid end to
// end and cut into equal shares, one a workgroup: every workgroup finds its own share
// from the lengths, so a long request among short ones costs no idle
// workgroups, and no host knows the lengths.  Waves take a row's tiles in turn
// and are joined in LDS.  A row cut between workgroups leaves its parts
// in the workspace, which swr_paged_join_kernel joins.
//
// What bounds it is K and V, read once: 2 requests of 262147 tokens (8 heads of 128 for
// 32, bf16) 391 to 395 us, 5.5 TB/s, where a copy reaches 5.2; 64 of 17 to 32768 tokens
// 225 to 231 us, 4.9 to 5.0 TB/s, of which 5 are the join.  Short rows are bound by the trips to memory,
// length, table, K, V: 4 requests of 300 to 700 tokens 12 us.  (With P in two parts, about 17 bits,
// 256 rows of 900 tokens took 22.9 us where they take 23.6, 2 requests of 262147 1 % less.)

constexpr int kTile = 32;      // tokens of a wave's tile
constexpr int kWaves = 4;
// Positions that a table (or a window) may have for its rows to be one block's each; the
// lengths are not known here.  (16 rows of 500 tokens, heads of 128, bf16:
// 9.9 us, 13.6 in shares, as they go in a wider table; of 1000 16.0 and 13.8, of 1500 20.7 and
// 14.2.  256 rows gain past it
// if they are alike, 1500 tokens 41 and 50, and lose if not, 17 to 2000 tokens 27.7 and 23.6.)
constexpr int kShort = 1024;
constexpr int64_t kMostRows = 1 << 23;   // (a launch has fewer than 2^32 threads, a row 512 of them)
// Shares of the work: three workgroups a compute unit, which is what a unit
// holds of heads of up to 256 bytes.  Not a power of two: of equal rows, whose
// lengths mostly are, shares would begin at multiples of large powers of two and so
// on few of the memory's channels (2 requests of 262147 tokens, 16 heads of 64, bf16: 512
// shares 476 us, 768 419, 1024 416; 8 heads of 128: 425, 396, 419).
constexpr int kShares = 768;
constexpr int kRowCost = 4;

// Tiles and first position of request b.
struct Rows {
    int64_t low;
    int tiles, length;
};
__device__ inline Rows rows_of(const PagedParams& p, int b) {
    const int64_t most = (int64_t)p.max_pages * p.page.d;
    const int64_t n = max(p.lengths[b], 0), low = p.window > 0 ? max(n - p.window, (int64_t)0) : 0;
    const int64_t end = min(n, most);   // (positions past the table are left out)
    return {low, end > low ? (int)((end - low + kTile - 1) / kTile) : 0, (int)end};
}

// The flat order: (request, head row within the request, place within the row).
// A row takes kRowCost places, in which nothing is done, before its tiles: what
// beginning and joining a row costs, in tiles, so that shares of many short rows are
// no longer than others (100 requests of 10 to 5000 tokens, 4 rows each: 45.3 us, with
// 0 places 61.8).
struct Place {
    int64_t total;   // places of all rows
    int64_t per;     // places a workgroup
    int b;           // the request that holds this workgroup's first place
    int64_t before;  // and the places before that request
};
__device__ inline int64_t places(const Rows& r, int heads) {
    return r.tiles ? (int64_t)(r.tiles + kRowCost) * heads : 0;
}

// Found by the whole block; buf holds 6 values.
__device__ inline Place find(const PagedParams& p, int heads, int64_t* buf) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t sum = 0;
    for (int b = threadIdx.x; b < p.batch; b += 256) sum += places(rows_of(p, b), heads);
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) buf[wave] = sum;
    __syncthreads();
    Place f;
    f.total = buf[0] + buf[1] + buf[2] + buf[3];
    f.per = max((f.total + p.workgroups - 1) / p.workgroups, (int64_t)(kWaves + kRowCost));
    const int64_t want = blockIdx.x * f.per;
    int64_t before = 0;
    f.b = p.batch;
    f.before = f.total;
    for (int c = 0; c < p.batch && want < f.total; c += 256) {
        const int b = c + (int)threadIdx.x;
        const int64_t n = b < p.batch ? places(rows_of(p, b), heads) : 0;
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

constexpr float kLowest = -3.402823466e38f;   // the least finite float

// A column's running maximum (the same on its four lanes) and this lane's sum
// of the weights against it.  The maximum is -infinity until a tile has a token, and
// from then on kLowest at least: tokens whose scores are all -infinity leave a sum of 0, and
// 0 / 0, but no token leaves y = 0.
struct Running {
    float m = -INFINITY, sum = 0.0f;

    // Scores (times log2 e) of a tile with or without any tokens to weights against the
    // running maximum; returns what the sums so far are multiplied by.
    __device__ float weigh(float (&p)[8], bool any) {
        float top = any ? fmaxf(m, kLowest) : m;
#pragma unroll
        for (int t = 0; t < 8; ++t) top = fmaxf(top, p[t]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.0f : top;   // (nothing yet: weights of 0, not NaN)
        const float alpha = __builtin_amdgcn_exp2f(m - base);
        m = top;
        float s = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            p[t] = __builtin_amdgcn_exp2f(p[t] - base);
            s += p[t];
        }
        sum = sum * alpha + s;
        return alpha;
    }
};

// Where a tile's 32 tokens lie: lane i % 32 has token i's row of the cache, in
// 16-byte units (0 where it has none), and every lane a bit for each that has one.
struct Spots {
    uint32_t row, valid;
    __device__ bool has(int t) const { return valid >> t & 1; }
};
constexpr uint32_t kAll = 0xffffffffu;

// One wave's state of one row: columns g = l.  A tile's K and V are loaded (load)
// and then worked in (use), so that one tile's loads may be on their way while
// another is worked on.  FULL: D is DP.  Tokens that are not there have the
// cache's first row loaded in their place, so that the loads stand without
// branches; their scores are replaced, and V's rows cleared, in the few tiles that
// have such.
template <class E, int DP, bool FULL>
struct State;

// bf16: DP = 32, 64, 128 or 256 channels (D rounded up).  Lane (l, u) holds
// channels 32 c + 8 u .. + 7 of K's token row l, and channels l * CH .. of V's rows.
template <int DP, bool FULL>
struct State<B16, DP, FULL> {
    static constexpr int CH = DP / 16;          // channels of V that a lane holds
    static constexpr int NK = DP / 32;
    struct Tile {
        u32x4 k[2][NK];
        uint32_t v[8][CH / 2];                  // token 16 (t / 4) + 4 u + t % 4
        uint32_t valid;
    };
    bf16x8 q[NK];
    f32x4 acc[CH];                              // acc[j]: channels (4 u + i) * CH + j, column l
    Running run;

    __device__ void begin(const uint16_t* qrow, bool in, int u, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            u32x4 v{0, 0, 0, 0};
            if (in && (FULL || 32 * c + 8 * u < D)) v = *(const u32x4*)(qrow + 32 * c + 8 * u);
            q[c] = __builtin_bit_cast(bf16x8, v);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) acc[j] = f32x4{0, 0, 0, 0};
    }

    __device__ static void load(Tile& x, const u32x4* kb, const u32x4* vb, const Spots& at, int l, int u, int D) {
        x.valid = at.valid;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const u32x4* k = kb + (uint32_t)__shfl((int)at.row, 16 * s + l) + u;
#pragma unroll
            for (int c = 0; c < NK; ++c) x.k[s][c] = FULL || 32 * c + 8 * u < D ? k[4 * c] : u32x4{0, 0, 0, 0};
        }
        const bool ok = FULL || l * CH < D;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t r = (uint32_t)__shfl((int)at.row, 16 * (t / 4) + 4 * u + t % 4);
            const uint32_t* v = (const uint32_t*)(vb + r) + l * (CH / 2);
            if constexpr (CH == 2) {
                x.v[t][0] = ok ? *v : 0;
            } else if constexpr (CH == 4) {
                const u32x2 w = ok ? *(const u32x2*)v : u32x2{0, 0};
                x.v[t][0] = w[0]; x.v[t][1] = w[1];
            } else {
#pragma unroll
                for (int h = 0; h < CH / 8; ++h) {
                    const u32x4 w = ok ? *(const u32x4*)(v + 4 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.v[t][4 * h + i] = w[i];
                }
            }
        }
    }

    __device__ void use(Tile& x, int u, float scale) {
        float p[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f32x4 d{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NK; ++c)
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[s][c]), q[c], d, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * s + i] = d[i] * scale;
        }
        if (x.valid != kAll) {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const bool in = x.valid >> (16 * (t / 4) + 4 * u + t % 4) & 1;
                if (!in) p[t] = -INFINITY;
#pragma unroll
                for (int j = 0; j < CH / 2; ++j)
                    if (!in) x.v[t][j] = 0;
            }
        }
        const float alpha = run.weigh(p, x.valid != 0);
        if (__any(alpha != 1.0f)) {   // (the maximum seldom moves)
#pragma unroll
            for (int j = 0; j < CH; ++j) acc[j] *= alpha;
        }
        bf16x8 w[3];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            // Cut off, not rounded: 8 bits each, and the differences are exact and not
            // negative.  The lower two are 2^-32 of the first at least (or the least bf16), far
            // below p's own rounding: a zero times an infinite value would be NaN where p's is
            // infinite.  A weight of 0 stays 0.
            const uint32_t a = __builtin_bit_cast(uint32_t, p[t]) & 0xffff0000u;
            const uint32_t least = a ? (uint32_t)max((int)a - (32 << 23), 0x10000) : 0;
            const float r = p[t] - as_float(a);
            const uint32_t b = __builtin_bit_cast(uint32_t, r) & 0xffff0000u;
            const uint32_t c = __builtin_bit_cast(uint32_t, r - as_float(b));
            w[0][t] = __builtin_bit_cast(__bf16, (uint16_t)(a >> 16));
            w[1][t] = __builtin_bit_cast(__bf16, (uint16_t)(max(b, least) >> 16));
            w[2][t] = __builtin_bit_cast(__bf16, (uint16_t)(max(c, least) >> 16));
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            // Channel l * CH + j of the lane's 8 tokens.
            u32x4 a;
#pragma unroll
            for (int t = 0; t < 4; ++t)
                a[t] = __builtin_amdgcn_perm(x.v[2 * t + 1][j / 2], x.v[2 * t][j / 2],
                                             j % 2 ? 0x07060302u : 0x05040100u);
            const bf16x8 v = __builtin_bit_cast(bf16x8, a);
#pragma unroll
            for (int i = 0; i < 3; ++i) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[i], acc[j], 0, 0, 0);
        }
    }
};

// float32: lane (l, u) holds channels 16 c + 4 u .. + 3 of K's token row l.
template <int DP, bool FULL>
struct State<B32, DP, FULL> {
    static constexpr int CH = DP / 16;
    static constexpr int NK = DP / 16;
    struct Tile {
        u32x4 k[2][NK];
        float v[8][CH];
        uint32_t valid;
    };
    f32x4 q[NK];
    f32x4 acc[CH];
    Running run;

    __device__ void begin(const float* qrow, bool in, int u, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            q[c] = f32x4{0, 0, 0, 0};
            if (in && (FULL || 16 * c + 4 * u < D)) q[c] = *(const f32x4*)(qrow + 16 * c + 4 * u);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) acc[j] = f32x4{0, 0, 0, 0};
    }

    __device__ static void load(Tile& x, const u32x4* kb, const u32x4* vb, const Spots& at, int l, int u, int D) {
        x.valid = at.valid;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const u32x4* k = kb + (uint32_t)__shfl((int)at.row, 16 * s + l) + u;
#pragma unroll
            for (int c = 0; c < NK; ++c) x.k[s][c] = FULL || 16 * c + 4 * u < D ? k[4 * c] : u32x4{0, 0, 0, 0};
        }
        const bool ok = FULL || l * CH < D;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t r = (uint32_t)__shfl((int)at.row, 16 * (t / 4) + 4 * u + t % 4);
            const uint32_t* v = (const uint32_t*)(vb + r) + l * CH;
            if constexpr (CH == 2) {
                const u32x2 w = ok ? *(const u32x2*)v : u32x2{0, 0};
                x.v[t][0] = as_float(w[0]); x.v[t][1] = as_float(w[1]);
            } else {
#pragma unroll
                for (int h = 0; h < CH / 4; ++h) {
                    const u32x4 w = ok ? *(const u32x4*)(v + 4 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.v[t][4 * h + i] = as_float(w[i]);
                }
            }
        }
    }

    __device__ void use(Tile& x, int u, float scale) {
        float p[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f32x4 d{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NK; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    d = __builtin_amdgcn_mfma_f32_16x16x4f32(as_float(x.k[s][c][i]), q[c][i], d, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * s + i] = d[i] * scale;
        }
        if (x.valid != kAll) {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const bool in = x.valid >> (16 * (t / 4) + 4 * u + t % 4) & 1;
                if (!in) p[t] = -INFINITY;
#pragma unroll
                for (int j = 0; j < CH; ++j)
                    if (!in) x.v[t][j] = 0.0f;
            }
        }
        const float alpha = run.weigh(p, x.valid != 0);
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int j = 0; j < CH; ++j) acc[j] *= alpha;
        }
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int j = 0; j < CH; ++j)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[t][j], p[t], acc[j], 0, 0, 0);
    }
};

__device__ inline void put(uint16_t* y, float f) { *y = __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ inline void put(float* y, float f) { *y = f; }

constexpr float kLn2 = 0.69314718055994530942f;

// Channel c of a row's output from its maximum, weighted sum and weights' sum; the
// maximum is -infinity where the row has no token.
template <class T>
__device__ inline void finish(const PagedParams& p, int b, int64_t head, int c, float m, float y, float sum) {
    if (c < p.D) put((T*)p.y + b * p.sy_b + head * p.sy_h + c, m == -INFINITY ? 0.0f : y / sum);
    if (c == 0 && p.lse)
        p.lse[(int64_t)b * p.kv_heads * p.group + head] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * kLn2;
}

// Floats of a row part in the workspace: 16 columns of DP channels, maxima, sums.
constexpr int64_t part_floats(int dp) { return 16 * ((int64_t)dp + 2); }

// Tiles t0 + wave, t0 + wave + WAVES, ... up to t1 of the row (request b, head
// row h) by the block's waves, and their parts joined in LDS.  Whole rows are
// finished; a part of one goes to `part`.
template <class E, int DP, int WAVES>
struct Joined {
    float m[WAVES][16], sum[WAVES][16];
    float acc[WAVES][DP][17];   // (17: the lanes' columns fall on different banks)
};

template <class E, int DP, bool FULL, int WAVES, bool AHEAD>
__device__ inline void attend(const PagedParams& p, const Rows& r, int b, int h, int t0, int t1, bool whole,
                              float* part, Joined<E, DP, WAVES>& join) {
    typedef typename E::T T;
    typedef State<E, DP, FULL> S;
    constexpr int CH = S::CH;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 16, u = lane / 16;
    const int kv = h / p.head_tiles, g0 = h % p.head_tiles * 16, columns = min(p.group - g0, 16);
    const int64_t head = (int64_t)kv * p.group + g0;
    const u32x4* kb = (const u32x4*)p.k + (int64_t)kv * p.s_head;
    const u32x4* vb = (const u32x4*)p.v + (int64_t)kv * p.s_head;
    const int32_t* table = p.table + b * p.st;
    // A tile's spots are looked up while the tile before it is worked on.
    const auto rows_at = [&](int t) {
        const int64_t pos = r.low + (int64_t)t * kTile + lane % kTile;
        Spots at{0, 0};
        bool in = t < t1 && pos < r.length;
        if (in) {
            const uint32_t page = p.page.over((uint32_t)pos);
            const int id = table[page];
            in = id >= 0 && id < p.pages;
            if (in) at.row = (uint32_t)id * p.s_page + ((uint32_t)pos - page * p.page.d) * p.s_token;
        }
        at.valid = (uint32_t)__ballot(in);
        return at;
    };
    Spots next = rows_at(t0 + wave);
    S s;
    s.begin((const T*)p.q + b * p.sq_b + (head + min(l, columns - 1)) * p.sq_h, l < columns, u, p.D);
    if constexpr (AHEAD) {
        // Two tiles in turn, one loaded while the other is worked in (a copy
        // from one to the other would wait for the loads).  What lies past t1 is
        // nothing, and adds nothing.
        typename S::Tile one, two;
        S::load(one, kb, vb, next, l, u, p.D);
        next = rows_at(t0 + wave + WAVES);
        for (int t = t0 + wave; t < t1; t += 2 * WAVES) {
            S::load(two, kb, vb, next, l, u, p.D);
            next = rows_at(t + 2 * WAVES);
            s.use(one, u, p.scale_log2);
            S::load(one, kb, vb, next, l, u, p.D);
            next = rows_at(t + 3 * WAVES);
            s.use(two, u, p.scale_log2);
        }
    } else {
        for (int t = t0 + wave; t < t1; t += WAVES) {
            typename S::Tile now;
            S::load(now, kb, vb, next, l, u, p.D);
            next = rows_at(t + WAVES);
            s.use(now, u, p.scale_log2);
        }
    }
    s.run.sum += __shfl_xor(s.run.sum, 16);
    s.run.sum += __shfl_xor(s.run.sum, 32);
    __syncthreads();   // (the last row's parts have been read)
    if (u == 0) { join.m[wave][l] = s.run.m; join.sum[wave][l] = s.run.sum; }
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) join.acc[wave][(4 * u + i) * CH + j][l] = s.acc[j][i];
    __syncthreads();
    for (int e = threadIdx.x; e < columns * DP; e += WAVES * 64) {
        const int g = e / DP, c = e % DP;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, join.m[w][g]);
        const float base = m == -INFINITY ? 0.0f : m;
        float y = 0.0f, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float a = __builtin_amdgcn_exp2f(join.m[w][g] - base);
            y += join.acc[w][c][g] * a;
            sum += join.sum[w][g] * a;
        }
        if (whole) {
            finish<T>(p, b, head + g, c, m, y, sum);
        } else {
            part[g * (DP + 2) + c] = y;
            if (c == 0) { part[g * (DP + 2) + DP] = m; part[g * (DP + 2) + DP + 1] = sum; }
        }
    }
}

// Rows without a token: zeros.
template <class T>
__device__ inline void nothing(const PagedParams& p, int b, int64_t head, int columns) {
    for (int e = threadIdx.x; e < columns * p.D; e += blockDim.x)
        finish<T>(p, b, head + e / p.D, e % p.D, -INFINITY, 0.0f, 0.0f);
}

// Waves of the kernel below that a SIMD holds (a compute unit as many blocks).
constexpr int waves_held(int head_bytes) { return head_bytes <= 256 ? 3 : 1; }

template <class E, int DP, bool FULL>
__global__ __launch_bounds__(kWaves * 64, waves_held(DP * sizeof(typename E::T))) void swr_paged_kernel(PagedParams p) {
    __shared__ int64_t buf[6];
    __shared__ Joined<E, DP, kWaves> join;
    const int heads = p.kv_heads * p.head_tiles;
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x)
        if (rows_of(p, b).tiles == 0) nothing<typename E::T>(p, b, 0, p.kv_heads * p.group);
    const Place f = find(p, heads, buf);
    const int64_t begin = blockIdx.x * f.per, end = min(begin + f.per, f.total);
    int4 cut = make_int4(0, 0, 0, 0);   // the row that begins here and goes on in the next shares
    int64_t at = begin, before = f.before;
    for (int b = f.b; at < end; ++b) {
        const Rows r = rows_of(p, b);
        if (r.tiles == 0) continue;
        const int length = r.tiles + kRowCost;
        for (int h = (int)((at - before) / length); h < heads && at < end; ++h) {
            const int64_t tile0 = before + (int64_t)h * length + kRowCost;   // the place of the row's first tile
            const int t0 = (int)max(at - tile0, (int64_t)0), t1 = (int)min((int64_t)r.tiles, end - tile0);
            if (t0 < t1) {
                // Parts: slot 0 of a row that began in an earlier share, slot 1 of one that goes on.
                attend<E, DP, FULL, kWaves, false>(p, r, b, h, t0, t1, t0 == 0 && t1 == r.tiles,
                                             p.part + (blockIdx.x * 2 + (t0 == 0 ? 1 : 0)) * part_floats(DP), join);
                if (t0 == 0 && t1 < r.tiles)
                    cut = make_int4(b, h, (int)((tile0 + r.tiles - 1) / f.per) - (int)blockIdx.x + 1, 0);
            }
            at = tile0 + t1;
        }
        before += places(r, heads);
    }
    if (threadIdx.x == 0) ((int4*)p.cuts)[blockIdx.x] = cut;
}

// Rows of few tokens, each a block's of its own: no shares to find or to join.
// Eight waves, or four of heads past 128 channels, for their registers (256 rows of 900
// tokens: 256 channels of float32 209 us with eight, 106 with four, of bf16 52.9 and
// 51.0, though 16 rows of 500 take 16.2 and 17.8; 128 of float32 52 and 57).
constexpr int short_waves(int channels) { return channels > 128 ? 4 : 8; }

template <class E, int DP, bool FULL>
__global__ __launch_bounds__(short_waves(DP) * 64) void swr_paged_short_kernel(PagedParams p) {
    constexpr int WAVES = short_waves(DP);
    __shared__ Joined<E, DP, WAVES> join;
    const int heads = p.kv_heads * p.head_tiles;
    const int b = (int)(blockIdx.x / heads), h = (int)(blockIdx.x % heads);
    const Rows r = rows_of(p, b);
    if (r.tiles == 0) {
        const int g0 = h % p.head_tiles * 16;
        nothing<typename E::T>(p, b, (int64_t)(h / p.head_tiles) * p.group + g0, min(p.group - g0, 16));
        return;
    }
    attend<E, DP, FULL, WAVES, DP * sizeof(typename E::T) <= 256>(p, r, b, h, 0, r.tiles, true, nullptr, join);
}

// The row that begins in a workgroup's share and goes on past it, if there is
// one (cuts): its parts there and in the workgroups after it.  The block's teams
// of 128 threads take a channel of a column each and their share of the parts, 8 at a
// time, and are joined in LDS, all in a fixed order.
struct Sum {
    float m = -INFINITY, y = 0.0f, sum = 0.0f;
    __device__ void add(float pm, float py, float psum) {
        const float top = fmaxf(m, pm), base = top == -INFINITY ? 0.0f : top;
        const float a = __builtin_amdgcn_exp2f(m - base), z = __builtin_amdgcn_exp2f(pm - base);
        y = y * a + py * z;
        sum = sum * a + psum * z;
        m = top;
    }
};

// Few rows are found by a block each, many by the shares that they begin in (4 rows of
// 100000 tokens: 55.1 us, by shares 58.2; 800 of 1100 to 3000: 169.2, by shares 164.9).
__host__ __device__ inline bool by_row(int rows, int shares) { return rows < shares / 4; }

template <class E, int DP>
__global__ __launch_bounds__(1024) void swr_paged_join_kernel(PagedParams p) {
    typedef typename E::T T;
    __shared__ float buf[7][3][128];
    // blockIdx.x is the share, or, where rows are few, the row (many blocks can
    // then have a slice of it each, and few of them find nothing).
    const int heads = p.kv_heads * p.head_tiles, rows = p.batch * heads;
    int share = blockIdx.x;
    if (by_row(rows, p.workgroups)) {
        __shared__ int found;
        if (threadIdx.x == 0) found = -1;
        __syncthreads();
        for (int i = threadIdx.x; i < p.workgroups; i += blockDim.x) {
            const int4 c = ((const int4*)p.cuts)[i];
            if (c.z > 0 && c.x * heads + c.y == (int)blockIdx.x) found = i;
        }
        __syncthreads();
        share = found;
        if (share < 0) return;
    }
    const int4 cut = ((const int4*)p.cuts)[share];
    const int b = cut.x, h = cut.y, parts = cut.z;
    if (parts == 0) return;
    const int lane = threadIdx.x % 128, team = threadIdx.x / 128, teams = blockDim.x / 128;
    const int kv = h / p.head_tiles, g0 = h % p.head_tiles * 16, columns = min(p.group - g0, 16);
    const int64_t head = (int64_t)kv * p.group + g0;
    // Part w is slot 1 of this share, then slot 0 of the next ones.
    const float* base = p.part + (int64_t)share * 2 * part_floats(DP);
    for (int e0 = blockIdx.y * 128; e0 < columns * DP; e0 += gridDim.y * 128) {
        const int e = e0 + lane, g = min(e / DP, columns - 1), c = e % DP;
        Sum s;
        for (int w0 = team; w0 < parts; w0 += 8 * teams) {
            float m[8], y[8], sum[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int w = min(w0 + teams * k, parts - 1);
                const float* part = base + (w == 0 ? 1 : 2 * (int64_t)w) * part_floats(DP) + g * (DP + 2);
                m[k] = w0 + teams * k < parts ? part[DP] : -INFINITY;
                sum[k] = part[DP + 1];
                y[k] = part[c];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (w0 + teams * k < parts) s.add(m[k], y[k], sum[k]);
        }
        __syncthreads();   // (the last channels' sums have been read)
        if (team > 0) { buf[team - 1][0][lane] = s.m; buf[team - 1][1][lane] = s.y; buf[team - 1][2][lane] = s.sum; }
        __syncthreads();
        if (team == 0 && e < columns * DP) {
            for (int k = 0; k < teams - 1; ++k) s.add(buf[k][0][lane], buf[k][1][lane], buf[k][2][lane]);
            finish<T>(p, b, head + g, c, s.m, s.y, s.sum);
        }
    }
}

int padded(int64_t D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256; }

template <class E, int DP, bool FULL>
hipError_t go(const PagedParams& p, hipStream_t st) {
    if (p.workgroups == 0) {
        hipLaunchKernelGGL((swr_paged_short_kernel<E, DP, FULL>), dim3((unsigned)(p.batch * p.kv_heads * p.head_tiles)),
                           dim3(short_waves(DP) * 64), 0, st, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((swr_paged_kernel<E, DP, FULL>), dim3((unsigned)p.workgroups), dim3(kWaves * 64), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Two teams where a row has a few parts on average, up to eight where it has many (800
    // rows of 1100 to 3000 tokens 164.9 us, with eight 173.5; 4 rows of 100000 55.1, with two 61.6).
    const int rows = p.batch * p.kv_heads * p.head_tiles, shares = p.workgroups;
    const int teams = rows >= shares / 8 ? 2 : rows >= shares / 64 ? 4 : 8;
    const int slices = std::min((std::min(p.group, 16) * DP + 127) / 128, by_row(rows, shares) ? 32 : 4);
    const int blocks = by_row(rows, shares) ? rows : shares;
    hipLaunchKernelGGL((swr_paged_join_kernel<E, DP>), dim3((unsigned)blocks, (unsigned)slices), dim3(128 * teams), 0,
                       st, p);
    return hipGetLastError();
}

template <class E, int DP>
hipError_t by_fill(const PagedParams& p, hipStream_t st) {
    return p.D == DP ? go<E, DP, true>(p, st) : go<E, DP, false>(p, st);
}

template <class E>
hipError_t by_width(const PagedParams& p, hipStream_t st) {
    switch (padded(p.D)) {
        case 32: return by_fill<E, 32>(p, st);
        case 64: return by_fill<E, 64>(p, st);
        case 128: return by_fill<E, 128>(p, st);
        default: return by_fill<E, 256>(p, st);
    }
}

}  // namespace

int paged_workgroups(const swr_paged_t& p) {
    const int64_t table = p.max_pages * p.cache.page_size;
    const int64_t positions = p.window > 0 ? std::min(p.window, table) : table;
    const int64_t heads = p.cache.heads * ((p.q_heads / p.cache.heads + 15) / 16);
    if (positions <= kShort && p.batch * heads < kMostRows) return 0;
    const double tiles = (double)p.batch * (double)heads * (double)((positions + kTile - 1) / kTile);
    return (int)std::min((double)kShares, (tiles + kWaves - 1) / kWaves);
}

int64_t paged_work_floats(const swr_paged_t& p) {
    return (int64_t)paged_workgroups(p) * (2 * part_floats(padded(p.cache.D)) + 4);
}

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
