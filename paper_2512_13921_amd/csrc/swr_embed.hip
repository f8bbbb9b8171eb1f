// swr_embed.hip -- rows of an embedding table, and the table's gradient, on gfx950.
//
//     y[i] = scale table[tokens[i]];      dtable[v] = scale sum over tokens[i] = v of dy[i]
//
// The forward moves its rows once.  The gradient sorts the positions by their tokens
// (a radix sort, or for up to 4096 counts for each; equal ones keep their order), so that a token's rows of dy are
// added in order by one thread, without atomics, and its row of the gradient is written once.
// The sorted positions are cut into windows of 16: a token's rows within one are
// summed in registers; sums that go on over a window's ends are kept as parts and
// joined in order.  The gradient's rows are all set to zero beforehand, by further blocks of the sort's own
// launches, which have little to do otherwise.
//
// What bounds it is the bytes: dy read once and the whole table written.  20495 tokens of 65536 x 2048 bf16 take 107 us: 52
// for the sort with the 268 MB of zeros (5.1 TB/s), 41 for the windows, 14 for the joins.
#include <algorithm>

#include "swr_lm_launch.h"
#include "swr_vectors.h"

namespace swr {
namespace {

constexpr int kSortThreads = 1024, kKeys = 4, kTileKeys = kSortThreads * kKeys;
constexpr int kBits = 9, kDigits = 1 << kBits;   // of a pass: two for 262143 tokens
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kWindow = 16;
constexpr int64_t kMostBlocks = 1 << 20;
constexpr int64_t kSummed = 64;   // tiles whose counts the scatter adds up by itself

unsigned grid_of(int64_t blocks) { return (unsigned)std::max<int64_t>(1, std::min(blocks, kMostBlocks)); }

// Threads of a block of 256 that take a row (or window): a power of two.
int row_shift(int64_t vectors) {
    int s = 0;
    while (s < 8 && ((int64_t)1 << s) < vectors) ++s;
    return s;
}

template <class E>
__global__ __launch_bounds__(256) void swr_embed_kernel(EmbedParams p, int shift) {
    typedef typename E::store T;
    const int t = threadIdx.x & ((1 << shift) - 1);
    const int64_t per_block = 256 >> shift;
    for (int64_t row = blockIdx.x * per_block + (threadIdx.x >> shift); row < p.rows; row += gridDim.x * per_block) {
        const int64_t token = p.wide_tokens ? ((const int64_t*)p.tokens)[row] : ((const int32_t*)p.tokens)[row];
        const bool there = token >= 0 && token < p.vocab;
        const T* in = (const T*)p.in + (there ? token : 0) * p.s_in;
        T* out = (T*)p.out + row * p.s_out;
        for (int64_t e = (int64_t)t * E::NE; e < p.width; e += (int64_t)E::NE << shift) {
            const int n = (int)(p.width - e);
            float f[E::NE] = {};
            if (there) {
                Slice<E, E::NE> s;
                s.load(in, (int)e, (int)p.width);
#pragma unroll
                for (int i = 0; i < E::NE; ++i) f[i] = s[i] * p.scale;
            }
            store<E, E::NE>(out + e, n, f);
        }
    }
}

// The sort's arrays within the workspace.
struct Sort {
    uint32_t *keys[2], *places[2];
    uint32_t* counts;          // [digit][tile]
    float* parts;              // [window][2][width]
    int64_t rows, tiles, windows;
    int bits, passes;
};
Sort layout(int64_t rows, int64_t vocab, void* work) {
    Sort s = {};
    s.rows = rows;
    s.tiles = (rows + kTileKeys - 1) / kTileKeys;
    s.windows = (rows + kWindow - 1) / kWindow;
    while (((int64_t)1 << s.bits) <= vocab) ++s.bits;   // (vocab stands for a token that is none)
    s.passes = (s.bits + kBits - 1) / kBits;
    char* w = (char*)work;
    const auto take = [&](int64_t bytes) {
        char* at = w;
        w += (bytes + 15) / 16 * 16;
        return at;
    };
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = (uint32_t*)take(rows * 4);
        s.places[i] = (uint32_t*)take(rows * 4);
    }
    s.counts = (uint32_t*)take(s.tiles * kDigits * 4);
    s.parts = (float*)w;
    return s;
}

__device__ inline uint32_t key_of(const EmbedParams& p, int64_t i) {
    const int64_t token = p.wide_tokens ? ((const int64_t*)p.tokens)[i] : ((const int32_t*)p.tokens)[i];
    return token >= 0 && token < p.vocab ? (uint32_t)token : (uint32_t)p.vocab;
}

// Rows first .. last - 1 of the gradient set to zero by blocks block, block + blocks, ...
template <class OE>
__device__ inline void clear_rows(const EmbedParams& p, int64_t first, int64_t last, int64_t block, int64_t blocks) {
    typedef typename OE::store T;
    const float zeros[OE::NE] = {};
    const int64_t vectors = (p.width + OE::NE - 1) / OE::NE;
    if (p.s_out == p.width) {   // one run of elements
        T* out = (T*)p.out + first * p.width;
        const int64_t n = (last - first) * p.width;
        for (int64_t e = (block * blockDim.x + threadIdx.x) * OE::NE; e < n; e += blocks * blockDim.x * OE::NE)
            store<OE, OE::NE>(out + e, (int)min(n - e, (int64_t)OE::NE), zeros);
        return;
    }
    for (int64_t row = first + block; row < last; row += blocks)
        for (int64_t v = threadIdx.x; v < vectors; v += blockDim.x)
            store<OE, OE::NE>((T*)p.out + row * p.s_out + v * OE::NE, (int)(p.width - v * OE::NE), zeros);
}

// Which rows of the gradient a launch of the sort clears: the share number `part` of `parts`.
struct Clear {
    int64_t sorting;   // the launch's blocks that sort; those after them clear
    int part, parts;
};
template <class OE>
__device__ inline bool clears(const EmbedParams& p, const Clear& c) {
    if (blockIdx.x < c.sorting) return false;
    const int64_t each = (p.vocab + c.parts - 1) / c.parts, first = min(each * c.part, p.vocab);
    clear_rows<OE>(p, first, min(first + each, p.vocab), blockIdx.x - c.sorting, gridDim.x - c.sorting);
    return true;
}

// A tile's keys of one digit: each thread's places among the equal ones before it in its wave
// (`rank`), and the waves' counts in LDS.  Keys are in order of rounds, lanes within them, waves apart.
__device__ inline void count_digits(const uint32_t* digit, const bool* there, uint32_t (*count)[kDigits], uint32_t* rank) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        uint64_t same = __ballot(there[k]);
#pragma unroll
        for (int bit = 0; bit < kBits; ++bit) {
            const bool on = digit[k] >> bit & 1;
            const uint64_t with = __ballot(on);
            same &= on ? with : ~with;
        }
        const uint32_t before = __popcll(same & (((uint64_t)1 << lane) - 1));
        uint32_t so_far = 0;
        if (there[k]) so_far = count[wave][digit[k]];
        rank[k] = so_far + before;
        if (there[k] && before == 0) count[wave][digit[k]] = so_far + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (read by other lanes of the wave in the next round)
    }
}

// In place of the waves' counts those of the waves before.
__device__ inline void sum_waves(uint32_t (*count)[kDigits]) {
    if (threadIdx.x < kDigits) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = count[w][threadIdx.x];
            count[w][threadIdx.x] = sum;
            sum += c;
        }
    }
}

// In place of a digit's values in LDS the sums of those before each; called by all threads of a block of kSortThreads.
__device__ inline void sum_digits(uint32_t* v) {
    __shared__ uint32_t totals[kDigits / 64];
    const int t = threadIdx.x, lane = t % 64, wave = t / 64;
    uint32_t own = 0, sum = 0;
    if (t < kDigits) {
        own = sum = v[t];
#pragma unroll
        for (int reach = 1; reach < 64; reach *= 2) {
            const uint32_t add = __shfl_up(sum, reach);
            if (lane >= reach) sum += add;
        }
        if (lane == 63) totals[wave] = sum;
    }
    __syncthreads();
    if (t < kDigits) {
        for (int w = 0; w < wave; ++w) sum += totals[w];
        v[t] = sum - own;
    }
    __syncthreads();
}

// Up to one tile of positions: each one's place is the number of smaller tokens, and of equal ones before it.  A block
// has 64 positions, one a lane, and its waves a part of the tokens each, which all blocks read.
// (A radix sort by one block took 12.5 us for 1001 tokens of 5003 with the gradient's 20 MB of zeros, this takes 6.7; 4096
// tokens of 65536 take 12.)
constexpr int kRankThreads = 1024, kRanked = 64;
template <class OE>
__global__ __launch_bounds__(kRankThreads) void swr_embed_sort_kernel(EmbedParams p, Sort s, Clear c) {
    constexpr int kWaves = kRankThreads / 64;
    __shared__ __attribute__((aligned(16))) uint32_t keys[kTileKeys];
    __shared__ uint32_t counts[kWaves][64];
    if (clears<OE>(p, c)) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = (int)s.rows, padded = (n + 63) / 64 * 64;
#pragma unroll 4
    for (int i = threadIdx.x; i < padded; i += kRankThreads) keys[i] = i < n ? key_of(p, i) : ~0u;
    __syncthreads();
    const int own = blockIdx.x * kRanked + lane;   // (of at most padded)
    const uint32_t key = keys[own];
    // Tokens in blocks of 64: of those before the positions' own equal ones count, of those behind it not.
    uint32_t count = 0;
    for (int block = wave; block < padded / 64; block += kWaves) {
        const uint32_t up_to = block < (int)blockIdx.x ? key + 1 : key;   // (a key is less than 2^31)
        const uint4* v = (const uint4*)(keys + block * 64);
        if (block != (int)blockIdx.x) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                count += (v[i].x < up_to) + (v[i].y < up_to) + (v[i].z < up_to) + (v[i].w < up_to);
        } else {
#pragma unroll 4
            for (int i = 0; i < 64; ++i) {
                const uint32_t other = keys[block * 64 + i];
                count += other < key || (other == key && i < lane);
            }
        }
    }
    counts[wave][lane] = count;
    __syncthreads();
    if (wave == 0 && own < n) {
#pragma unroll
        for (int w = 1; w < kWaves; ++w) count += counts[w][lane];
        s.keys[s.passes % 2][count] = key;
        s.places[s.passes % 2][count] = own;
    }
}

// Counts of a pass's digits, tile by tile.
template <class OE>
__global__ __launch_bounds__(kSortThreads) void swr_embed_count_kernel(EmbedParams p, Sort s, Clear c, int pass) {
    __shared__ uint32_t count[kDigits];
    if (clears<OE>(p, c)) return;
    const uint32_t* keys = s.keys[pass % 2];
    for (int64_t tile = blockIdx.x; tile < s.tiles; tile += c.sorting) {
        if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kKeys; ++k) {
            const int64_t i = tile * kTileKeys + k * kSortThreads + threadIdx.x;
            if (i < s.rows) atomicAdd(&count[(pass ? keys[i] : key_of(p, i)) >> kBits * pass & (kDigits - 1)], 1u);
        }
        __syncthreads();
        if (threadIdx.x < kDigits) s.counts[threadIdx.x * s.tiles + tile] = count[threadIdx.x];
        __syncthreads();
    }
}

// In place of a digit's counts those of the tiles before (for many tiles), and the digit's total in the place
// of its last tile's: a block a digit.
constexpr int kScanThreads = 256;
__global__ __launch_bounds__(kScanThreads) void swr_embed_scan_kernel(Sort s) {
    __shared__ uint32_t sums[kScanThreads];
    __shared__ uint32_t carry;
    uint32_t* counts = s.counts + (int64_t)blockIdx.x * s.tiles;
    if (threadIdx.x == 0) carry = 0;
    for (int64_t first = 0; first < s.tiles; first += kScanThreads) {
        const int64_t i = first + threadIdx.x;
        const uint32_t own = i < s.tiles ? counts[i] : 0;
        __syncthreads();
        sums[threadIdx.x] = own;
        __syncthreads();
        for (int reach = 1; reach < kScanThreads; reach *= 2) {
            const uint32_t add = (int)threadIdx.x >= reach ? sums[threadIdx.x - reach] : 0;
            __syncthreads();
            sums[threadIdx.x] += add;
            __syncthreads();
        }
        if (i < s.tiles) counts[i] = carry + sums[threadIdx.x];   // (of the tiles up to this one)
        __syncthreads();
        if (threadIdx.x == 0) carry += sums[kScanThreads - 1];
    }
}

// One pass: a tile's keys to their places in the order of the pass's digit.
template <class OE>
__global__ __launch_bounds__(kSortThreads) void swr_embed_scatter_kernel(EmbedParams p, Sort s, Clear c, int pass,
                                                                         bool scanned) {
    __shared__ uint32_t count[kSortWaves][kDigits], base[kDigits], mine[kDigits];
    if (clears<OE>(p, c)) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t *keys = s.keys[pass % 2], *places = s.places[pass % 2];
    uint32_t *to_keys = s.keys[(pass + 1) % 2], *to_places = s.places[(pass + 1) % 2];
    for (int64_t tile = blockIdx.x; tile < s.tiles; tile += c.sorting) {
        for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) (&count[0][0])[i] = 0;
        // Of each digit: the keys in the tiles before, and in all of them.
        if (threadIdx.x < kDigits) {
            const uint32_t* counts = s.counts + (int64_t)threadIdx.x * s.tiles;
            uint32_t before = 0, all = 0;
            if (scanned) {
                before = tile ? counts[tile - 1] : 0;
                all = counts[s.tiles - 1];
            } else {
                for (int64_t i = 0; i < s.tiles; ++i) {
                    const uint32_t n = counts[i];
                    if (i < tile) before += n;
                    all += n;
                }
            }
            mine[threadIdx.x] = before;
            base[threadIdx.x] = all;
        }
        __syncthreads();
        sum_digits(base);
        uint32_t key[kKeys], place[kKeys], digit[kKeys], rank[kKeys];
        bool there[kKeys];
#pragma unroll
        for (int k = 0; k < kKeys; ++k) {
            const int64_t i = tile * kTileKeys + wave * 64 * kKeys + k * 64 + lane;
            there[k] = i < s.rows;
            key[k] = place[k] = 0;
            if (there[k]) {
                key[k] = pass ? keys[i] : key_of(p, i);
                place[k] = pass ? places[i] : (uint32_t)i;
            }
            digit[k] = key[k] >> kBits * pass & (kDigits - 1);
        }
        count_digits(digit, there, count, rank);
        __syncthreads();
        sum_waves(count);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kKeys; ++k) {
            if (!there[k]) continue;
            const int64_t to = (int64_t)base[digit[k]] + mine[digit[k]] + count[wave][digit[k]] + rank[k];
            to_keys[to] = key[k];
            to_places[to] = place[k];
        }
        __syncthreads();
    }
}

// Sums over the windows of the sorted positions.  Rows of tokens that begin and end in the window are
// written; the sum of a token that comes from the window before is its part 0, that of
// one that begins here and goes on its part 1.
//
// WHOLE: rows of a vector and more; the last one of a row ends with it, and writes some elements once more, the same.
// (With branches for its elements the code is long, and few tokens wait for it to be fetched: 8.5 us for 1001
// of 1001 float32, this 6.2; 20495 of 2048 bf16 take 41 either way.)
template <class E, class OE, bool WHOLE>
__global__ __launch_bounds__(256) void swr_embed_window_kernel(EmbedParams p, Sort s, int shift) {
    typedef typename E::store T;
    constexpr int NE = E::NE, kAhead = 8;
    const uint32_t *keys = s.keys[s.passes % 2], *places = s.places[s.passes % 2];
    const int t = threadIdx.x & ((1 << shift) - 1);
    const int64_t per_block = 256 >> shift;
    for (int64_t w = blockIdx.x * per_block + (threadIdx.x >> shift); w < s.windows; w += gridDim.x * per_block) {
        const int64_t first = w * kWindow;
        const int n = (int)min((int64_t)kWindow, s.rows - first);
        const uint32_t before = first ? keys[first - 1] : ~0u, after = first + n < s.rows ? keys[first + n] : ~0u;
        for (int64_t column = ((int64_t)blockIdx.y << shift) * NE + (int64_t)t * NE; column < p.width;
             column += ((int64_t)gridDim.y << shift) * NE) {
            const int64_t e = WHOLE ? min(column, p.width - NE) : column;
            const int left = WHOLE ? NE : (int)min(p.width - e, (int64_t)NE);
            float sum[NE] = {};
            uint32_t token = keys[first];
            bool comes = token == before;
            for (int i = 0; i < n; i += kAhead) {
                uint32_t key[kAhead], place[kAhead];
                Slice<E, NE> row[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    key[k] = i + k < n ? keys[first + i + k] : ~0u;
                    place[k] = i + k < n ? places[first + i + k] : 0;
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    row[k] = {};
                    if (key[k] < p.vocab) row[k].load((const T*)p.in + place[k] * p.s_in + e, 0, left);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (i + k >= n) break;
                    if (key[k] != token) {
                        if (token < p.vocab) {
                            if (comes) {
                                store<F32, NE>(s.parts + (2 * w) * p.width + e, left, sum);
                            } else {
                                float f[NE];
#pragma unroll
                                for (int c = 0; c < NE; ++c) f[c] = sum[c] * p.scale;
                                store<OE, NE>((typename OE::store*)p.out + token * p.s_out + e, left, f);
                            }
                        }
                        token = key[k];
                        comes = false;
#pragma unroll
                        for (int c = 0; c < NE; ++c) sum[c] = 0.0f;
                    }
#pragma unroll
                    for (int c = 0; c < NE; ++c) sum[c] += row[k][c];
                }
            }
            if (token < p.vocab) {
                if (comes || token == after) {
                    store<F32, NE>(s.parts + (2 * w + !comes) * p.width + e, left, sum);
                } else {
#pragma unroll
                    for (int c = 0; c < NE; ++c) sum[c] *= p.scale;
                    store<OE, NE>((typename OE::store*)p.out + token * p.s_out + e, left, sum);
                }
            }
        }
    }
}

// Sums of tokens that go on over windows' ends, each by the window that it begins in: that
// window's part 1 and the part 0 of those that begin with the same token.  A block's four waves take a quarter of
// them each, one after the other, 64 vectors of 4 columns, and their sums are added in order.
constexpr int kJoinVectors = 2;   // of a lane
template <class OE>
__global__ __launch_bounds__(256) void swr_embed_join_kernel(EmbedParams p, Sort s) {
    constexpr int NE = 4;
    __shared__ float sums[3][kJoinVectors * NE][64];
    const uint32_t* keys = s.keys[s.passes % 2];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int64_t w = blockIdx.x; w + 1 < s.windows; w += gridDim.x) {
        const int64_t first = w * kWindow;
        const uint32_t token = keys[first + kWindow - 1];
        // (it goes on, and begins in this window)
        if (token >= p.vocab || keys[first + kWindow] != token || (first && keys[first - 1] == token)) continue;
        // The last window that begins with the token.
        int64_t low = w + 1, high = s.windows;
        while (high - low > 1) {
            const int64_t mid = (low + high) / 2;
            if (keys[mid * kWindow] == token) low = mid;
            else high = mid;
        }
        // Parts 0 .. low - w: this window's part 1, then the others' part 0.
        const int64_t parts = low - w + 1, each = (parts + 3) / 4, begin = min(wave * each, parts), end = min(begin + each, parts);
        for (int64_t base = (int64_t)blockIdx.y * 64 * kJoinVectors * NE; base < p.width;
             base += (int64_t)gridDim.y * 64 * kJoinVectors * NE) {
            float sum[kJoinVectors][NE] = {};
#pragma unroll 4
            for (int64_t k = begin; k < end; ++k) {
                const float* row = s.parts + (k == 0 ? 2 * w + 1 : 2 * (w + k)) * p.width;
#pragma unroll
                for (int v = 0; v < kJoinVectors; ++v) {
                    const int64_t e = base + (v * 64 + lane) * NE;
                    Slice<F32, NE> f;
                    f.load(row, (int)min(e, p.width), (int)p.width);
#pragma unroll
                    for (int c = 0; c < NE; ++c) sum[v][c] += f[c];
                }
            }
            if (wave > 0) {
#pragma unroll
                for (int i = 0; i < kJoinVectors * NE; ++i) sums[wave - 1][i][lane] = sum[i / NE][i % NE];
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int v = 0; v < kJoinVectors; ++v) {
                    const int64_t e = base + (v * 64 + lane) * NE;
                    typename OE::store* out = (typename OE::store*)p.out + token * p.s_out + e;
#pragma unroll
                    for (int c = 0; c < NE; ++c) {
#pragma unroll
                        for (int g = 0; g < 3; ++g) sum[v][c] += sums[g][v * NE + c][lane];
                        if (e + c < p.width) out[c] = OE::to(sum[v][c] * p.scale);
                    }
                }
            }
            __syncthreads();
        }
    }
}

template <class E, class OE>
hipError_t backward(const EmbedParams& p, void* work, hipStream_t st) {
    const Sort s = layout(p.rows, p.vocab, work);
    hipError_t e;
    // Blocks that clear, a launch: 32 KB each, at most what the GPU holds.
    const int64_t bytes = p.vocab * p.width * (int64_t)sizeof(typename OE::store);
    const auto clearing = [&](int parts) {
        return std::max<int64_t>(1, std::min<int64_t>(480, bytes / parts / 32768));
    };
    if (p.rows == 0 || s.tiles == 1) {
        const Clear c{(p.rows + kRanked - 1) / kRanked, 0, 1};
        hipLaunchKernelGGL((swr_embed_sort_kernel<OE>), dim3((unsigned)(c.sorting + clearing(1))), dim3(kRankThreads), 0,
                           st, p, s, c);
        if ((e = hipGetLastError()) != hipSuccess || p.rows == 0) return e;
    } else {
        const bool scanned = s.tiles > kSummed;
        const int parts = 2 * s.passes;
        const int64_t blocks = std::min(s.tiles, kMostBlocks);
        const unsigned grid = (unsigned)(blocks + clearing(parts));
        for (int pass = 0; pass < s.passes; ++pass) {
            hipLaunchKernelGGL((swr_embed_count_kernel<OE>), dim3(grid), dim3(kSortThreads), 0, st, p, s,
                               Clear{blocks, 2 * pass, parts}, pass);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            if (scanned) {
                hipLaunchKernelGGL(swr_embed_scan_kernel, dim3(kDigits), dim3(kScanThreads), 0, st, s);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
            hipLaunchKernelGGL((swr_embed_scatter_kernel<OE>), dim3(grid), dim3(kSortThreads), 0, st, p, s,
                               Clear{blocks, 2 * pass + 1, parts}, pass, scanned);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    const auto columns = [&](int ne, int shift) {
        return (unsigned)std::max<int64_t>(1, std::min<int64_t>(1024, (p.width + ((int64_t)ne << shift) - 1) /
                                                                           ((int64_t)ne << shift)));
    };
    const int shift = row_shift((p.width + E::NE - 1) / E::NE);
    const int64_t per_block = 256 >> shift;
    const auto window = p.width >= E::NE ? swr_embed_window_kernel<E, OE, true> : swr_embed_window_kernel<E, OE, false>;
    hipLaunchKernelGGL(window,
                       dim3(grid_of((s.windows + per_block - 1) / per_block), columns(E::NE, shift)), dim3(256), 0, st,
                       p, s, shift);
    if ((e = hipGetLastError()) != hipSuccess || s.windows == 1) return e;
    hipLaunchKernelGGL((swr_embed_join_kernel<OE>),
                       dim3(grid_of(s.windows), (unsigned)std::min<int64_t>(1024, (p.width + 256 * kJoinVectors - 1) /
                                                                                      (256 * kJoinVectors))),
                       dim3(256), 0, st, p, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(int dtype, const EmbedParams& p, void* stream) {
    const int ne = dtype == SWR_DTYPE_F32 ? F32::NE : Bf16::NE, shift = row_shift((p.width + ne - 1) / ne);
    const unsigned grid = grid_of((p.rows + (256 >> shift) - 1) / (256 >> shift));
    if (dtype == SWR_DTYPE_F32)
        hipLaunchKernelGGL((swr_embed_kernel<F32>), dim3(grid), dim3(256), 0, (hipStream_t)stream, p, shift);
    else
        hipLaunchKernelGGL((swr_embed_kernel<Bf16>), dim3(grid), dim3(256), 0, (hipStream_t)stream, p, shift);
    return hipGetLastError();
}

int64_t embed_work_bytes(int64_t rows, int64_t vocab, int64_t width) {
    if (rows == 0) return 0;
    const Sort s = layout(rows, vocab, nullptr);
    return (int64_t)(uintptr_t)s.parts + s.windows * 2 * width * 4;
}

hipError_t launch_embed_backward(int dtype, int out_dtype, const EmbedParams& p, void* work, void* stream) {
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == SWR_DTYPE_F32) return backward<F32, F32>(p, work, st);
    return out_dtype == SWR_DTYPE_F32 ? backward<Bf16, F32>(p, work, st) : backward<Bf16, Bf16>(p, work, st);
}

}  // namespace swr
