// swr_hybrid_launch.h -- internal interface between the host API of the
// hybrid model's operators (swr_hybrid_api.cpp) and their gfx950 kernels
// (swr_norm.hip, swr_fp4.hip, swr_paged.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/swr_hybrid.h"

namespace swr {

// Norm: everything validated by the host.  Row r is (r / inner, r % inner).
struct NormParams {
    const void* x;       // forward: x; backward: h
    const void* r;       // forward: residual or NULL; backward: dh or NULL
    const void* w;
    void* y;             // forward: y; backward: dy (read)
    void* h;             // forward: h or NULL; backward: dx
    float* scale;        // [rows], out_dtype FP8
    float* dw;           // [width]
    float* partial;      // [blocks][width]: the blocks' shares of dw
    float2* stats;       // [rows]: 1 / rms and mean(g n) / rms^2 of wide rows (backward)
    int64_t rows;
    uint32_t inner;
    int32_t width;
    float eps;
    int64_t sx_o, sx_i, sr_o, sr_i, sh_o, sh_i, sy_o, sy_i;
};

// How a norm launch covers its rows: a row by a wave (blocks of four) or by a
// block of its own, vpt 16-byte vectors of it in a thread's registers (vpt = 0:
// rows too wide for that, walked twice).
struct NormPlan {
    bool block;
    int vpt, threads;
    int blocks;          // backward: workgroups, each with a share of dw
};
NormPlan plan_norm(int dtype, int64_t rows, int64_t width, bool backward);
hipError_t launch_norm(const swr_norm_t& n, const NormPlan& plan, const NormParams& p, void* stream);
hipError_t launch_norm_backward(const swr_norm_t& n, const NormPlan& plan, const NormParams& p, void* stream);

struct Fp4Params {
    const void* x;
    const float* scale;
    const uint8_t* codes;
    const uint8_t* powers;
    void* y;
    int32_t M, N, K;
    int64_t sx, sy, sc, sp;
    int32_t m_blocks;    // the launch's: blocks along M
};
hipError_t launch_fp4(int dtype, int out_dtype, const Fp4Params& p, void* stream);
hipError_t launch_fp4_pack(int dtype, const void* w, int64_t N, int64_t K, int64_t sw, uint8_t* codes, uint8_t* powers,
                           int64_t sc, int64_t sp, void* stream);

// Division of whole numbers below 2^31 by d (1 to 65536) with a multiplication:
// with L = ceil(log2 d) and m = floor(2^(31 + L) / d) + 1 < 2^32, n m exceeds
// n 2^(31 + L) / d by less than 2^(31 + L) / d.
struct Divisor {
    uint32_t d, m, shift;   // m = 0: d is 1
    Divisor() = default;
    explicit Divisor(int64_t by) : d((uint32_t)by), m(0), shift(0) {
        if (by <= 1) return;
        uint32_t L = 0;
        while (((int64_t)1 << L) < by) ++L;
        m = (uint32_t)(((uint64_t)1 << (31 + L)) / d + 1);
        shift = L - 1;
    }
    __device__ uint32_t over(uint32_t n) const { return m ? __umulhi(n, m) >> shift : n; }
};

struct TableParams {
    const int32_t *lengths, *news, *stack, *count;
    int32_t* table;
    int64_t* slots;
    int32_t *starts, *new_lengths, *new_count;
    int32_t batch, max_pages, page_size, free_pages;
    int64_t st, tokens;
    Divisor page;                        // by the page size
};
hipError_t launch_tables(const TableParams& p, void* stream);

// Cache strides here are in 16-byte units.
struct AppendParams {
    const void *k, *v;
    void *k_cache, *v_cache;
    const int64_t* slots;
    int64_t tokens, rows;                // rows: pages * page_size
    uint32_t page_size;
    uint32_t per_head, per_token;        // 16-byte vectors of a head's and of a token's channels
    int64_t sk_t, sk_h, sv_t, sv_h;
    int64_t s_page, s_token, s_head;
};
hipError_t launch_append(const AppendParams& p, void* stream);

struct PagedParams {
    const void *q, *k, *v;
    const int32_t *table, *lengths;
    void* y;
    float* lse;
    float* part;                         // parts of rows cut between workgroups: [workgroups][2][16][dp + 2]
    int32_t* cuts;                       // [workgroups][4]: request, head row and parts of such a row
    int32_t batch, kv_heads, group;      // group: query heads that share a key head
    int32_t head_tiles;                  // ceil(group / 16)
    int32_t D, max_pages, pages;
    Divisor page;                        // by the page size
    int32_t workgroups;                  // among which the tiles are shared out; 0: a workgroup a row
    int64_t st, window;
    int64_t sq_b, sq_h, sy_b, sy_h;      // elements
    uint32_t s_page, s_token, s_head;    // 16-byte units
    float scale_log2;                    // scale * log2(e)
};
// Workgroups that share out the attention's work (0: a workgroup a row).
int paged_workgroups(const swr_paged_t& p);
int64_t paged_work_floats(const swr_paged_t& p);
hipError_t launch_paged(int dtype, const PagedParams& p, void* stream);

}  // namespace swr
