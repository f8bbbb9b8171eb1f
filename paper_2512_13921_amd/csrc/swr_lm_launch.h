// swr_lm_launch.h -- internal interface between the host API of a recurrent
// language model's operators (swr_lm_api.cpp) and their gfx950 kernels
// (swr_embed.hip, swr_conv.hip, swr_scan.hip, swr_logprob.hip).  Not part of the
// public ABI; everything in these structs is validated by the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/swr_lm.h"

namespace swr {

struct EmbedParams {
    const void* tokens;
    bool wide_tokens;                    // int64, else int32
    const void* in;                      // table, or dy
    void* out;                           // y, or dtable
    int64_t rows, vocab, width;
    int64_t s_in, s_out;                 // row strides
    float scale;
};
hipError_t launch_embed(int dtype, const EmbedParams& p, void* stream);
int64_t embed_work_bytes(int64_t rows, int64_t vocab, int64_t width);
hipError_t launch_embed_backward(int dtype, int out_dtype, const EmbedParams& p, void* work, void* stream);

struct ConvParams {
    const void *x, *w, *bias, *state, *dy;
    const int32_t* lengths;
    void *y, *state_out, *dx;
    float *dw, *db, *partial;
    int64_t B, T, C;
    int64_t sx_b, sx_t, sy_b, sy_t, sd_b, sd_t;
    bool silu;
};
hipError_t launch_conv(int dtype, int taps, const ConvParams& p, void* stream);
int64_t conv_work_bytes(int64_t B, int64_t T, int64_t C, int taps);
hipError_t launch_conv_backward(int dtype, int taps, const ConvParams& p, void* stream);

// Channels of a block of threads, and runs of tokens that the work is cut into.
struct ScanPlan {
    int states;                          // of a channel, a lane: 4 or 1
    int lanes;                           // lanes that share a channel's states: a power of two
    int64_t chunk;                       // tokens of a run, a multiple of SWR_SCAN_BLOCK
    int64_t chunks;                      // runs of a sequence
    int64_t tiles;                       // blocks of channels of a group
    int64_t blocks(int64_t B, int64_t G) const { return B * G * tiles * chunks; }
};
ScanPlan plan_scan(const swr_scan_t& p, bool backward);

struct ScanParams {
    swr_scan_inputs_t in;
    const void* dy;
    const float *carriers_in, *dh_last;
    void* y;
    float *carriers, *h_last;
    swr_scan_gradients_t out;
    float* states;                       // [B][chunks][D][N]: a run's own states, then those that it starts from
    float* steps;                        // [B][chunks][D]: sums of a run's steps
    float* shares;                       // backward: [B][T][G][tiles][2][N], shares of dB and dC
    float* sums;                         // backward: [B][chunks][D][N + 2], shares of dA, dbias and dskip
    int64_t B, T, D, G, Dg;              // Dg: D / G
    int32_t N;
    bool softplus;
    int64_t sx_b, sx_t, sdt_b, sdt_t, sz_b, sz_t, sy_b, sy_t, sB_b, sB_t, sB_g, sC_b, sC_t, sC_g;
    int64_t chunk, chunks, tiles, work;  // work: blocks of threads that the plan asks for
};
int64_t scan_work_floats(const swr_scan_t& p, const ScanPlan& plan);
int64_t scan_backward_work_floats(const swr_scan_t& p, const ScanPlan& plan);
hipError_t launch_scan(int dtype, const ScanPlan& plan, const ScanParams& p, void* stream);
hipError_t launch_scan_backward(int dtype, const ScanPlan& plan, const ScanParams& p, void* stream);

struct LogProbParams {
    const void *logits, *tokens;
    bool wide_tokens;
    float *logp, *lse, *entropy, *top_logp;
    int64_t* top_tokens;
    const float *lse_in, *entropy_in, *dlogp, *dlse, *dentropy;
    void* dlogits;
    void* work;
    int64_t rows, vocab, sl, sd;
    int32_t top, parts;                  // parts: blocks that share a row
    float scale;
};
int logprob_parts(int64_t rows, int64_t vocab);
int64_t logprob_work_bytes(int64_t rows, int64_t vocab, int top);
hipError_t launch_logprob(int dtype, const LogProbParams& p, void* stream);
hipError_t launch_logprob_backward(int dtype, const LogProbParams& p, void* stream);

}  // namespace swr
