// Internal declarations of the operators for token models: rotary positions, attention with a decay for each head, log
// probabilities, the gated delta rule, layer norm, verification of drafts (rotary_kernels.hip, attention_kernels.hip, logprob_kernels.hip, delta_kernels.hip, norm_kernels.hip, verify_kernels.hip; host
// side in token_api.hip).
#pragma once

#include "laplex_internal.h"

namespace laplex {

constexpr int64_t kLogprobMaxRows = 0xFFFFFFFEll;          // logits of a column: their places are 32-bit

int hip_failed(hipError_t e);      // keeps the error's text for laplex_last_hip_error (api.hip)

// ----------------------------------------------------------------------------
// Rotary positions.
// ----------------------------------------------------------------------------
struct RotaryArgs {
    const void* x; void* y;
    int64_t ldx, ldy, tokens;
    int heads, dim, half;            // half = pairs of a head that are turned
    const int64_t* positions;
    const float* frequencies;
    float magnitude;
    bool bf16, interleaved, inverse;
};
hipError_t launch_rotary(const RotaryArgs& A, hipStream_t st);
hipError_t launch_rotary_frequencies(float* out, int64_t pairs, double base, int scaling, double factor, double context,
                                     double low, double high, hipStream_t st);

// ----------------------------------------------------------------------------
// Attention with a decay for each head.  A walk goes over the tokens of every sequence in one direction, u = 0, 1, ...:
//   out_u = out_scale * ( inner sum_{w <= u} l^(u - w) (q_u . k_w) v_w + l^(u + lead) q_u X ),      l = exp(-rate of the head)
//   last  = last_scale * ( l^n X + inner sum_w l^(n - w - lead) k_w v_w^T ),                        X = state_in / last_scale
// The forward call is one walk ahead (lead = 1), the backward call one ahead (gq) and two back (gk, gv: lead = 0), with the
// parts of q, k, v changed about; a state matrix is read transposed where those swap its two sides.
// ----------------------------------------------------------------------------
struct Walk {
    const void *q, *k, *v;
    void* out;                       // may be null: only `last` is wanted
    int64_t ldq, ldk, ldv, ldo;
    int dk, dv;                      // of this walk: the state is dk x dv
    int reverse, lead, transposed;   // transposed: state_in lies as dv x dk
    int exact;                       // the walk's state can be asked for: an fp32 sum of fp32 products, whether it is or not (so that `out` has the same bits)
    const float* state_in;           // [sequences][heads][dk][dv] (or [dv][dk]) or null
    float* state_out;                // the same, never transposed, or null
    float inner, out_scale, last_scale;
    int set, set_transposed;         // which of the state sets below holds the states that enter its stretches, and whether with its sides swapped
};

struct AttentionArgs {
    Walk walk[3];
    int walks;
    Walk states[2];                  // state sets: walks whose states alone are formed, where sequences are cut into stretches.  gk and gv share one
    int sets;
    const int64_t* starts;           // [sequences + 1] or null: equal lengths
    int64_t tokens, sequences;
    int heads;
    const float* rates;
    bool bf16, backward;
    char* ws;
    // filled in by launch_attention
    int64_t stretch, per_sequence, slots;   // tokens of a stretch that one workgroup walks; stretches of a sequence (equal lengths), of all, at most
    int64_t places;                  // states that enter stretches of sequences that have several, at most
    int slices;                      // workgroups side by side over the columns
    int wide[3], states_wide[2];     // per walk, a bit each for q, k, v, out: its rows may be accessed four numbers at a time
};
size_t attention_workspace(int64_t tokens, int64_t sequences, int heads, int dk, int dv);
hipError_t launch_attention(const AttentionArgs& A, hipStream_t st);

struct AttentionStepArgs {
    const void *q, *k, *v;
    void* y;
    int64_t ldq, ldk, ldv, ldy, sequences;
    int heads, dk, dv;
    const float* rates;
    float scale;
    float* state;                    // [sequences][heads][dk][dv]
    bool bf16;
};
hipError_t launch_attention_step(const AttentionStepArgs& A, hipStream_t st);

// ----------------------------------------------------------------------------
// Attention by the gated delta rule.
// ----------------------------------------------------------------------------
struct DeltaArgs {
    const void *q, *k, *v, *gy;
    void *y, *gq, *gk, *gv;          // gq, gk, gv: any may be null
    int64_t ldq, ldk, ldv, ldy, ldgy, ldgq, ldgk, ldgv;
    const float *rates, *beta;       // [tokens][heads], rows ldr and ldb apart
    float *grates, *gbeta;           // the same, either may be null
    int64_t ldr, ldb, ldgr, ldgb;
    int64_t tokens, sequences;
    const int64_t *starts, *lengths; // either may be null
    int heads, key_heads, dk, dv;
    float scale;
    const float *state_in, *gstate_out;      // [sequences][heads][dk][dv], any of the four may be null
    float *state_out, *gstate_in;
    bool bf16, forward, saved;       // saved: the forward call leaves, and the backward call finds, what the gradients need
    char* ws;
    // filled in by launch_delta
    int slices, wide;                // workgroups side by side over the columns; a bit each for q, k, v, y, gy, gq, gk: four numbers at a time
    int64_t each, per_sequence, chunks;      // tokens of a sequence (equal lengths); chunks of a sequence (equal lengths), of all, at most
    int64_t stretch, stretches, slots;       // tokens of a stretch that one workgroup walks; stretches of a sequence (equal lengths), of all, at most
    bool training;
    float *maps, *states_out, *u_out, *gstates, *r_out;
    float *added, *turned, *added_back;      // [place][head]: what a stretch adds to the state (then: the state that enters it), how it turns it, what it adds to the state's gradient
};
size_t delta_workspace(bool bf16, int64_t tokens, int64_t sequences, int heads, int dk, int dv, bool training);
hipError_t launch_delta(const DeltaArgs& A, hipStream_t st);
hipError_t launch_delta_tokens(const DeltaArgs& A, hipStream_t st);      // forward, for sequences of a few tokens

// ----------------------------------------------------------------------------
// Log probabilities over logits y[k][batch].
// ----------------------------------------------------------------------------
struct LogprobArgs {
    const void* y;
    int64_t ldy, k, batch;
    bool bf16;
    const int64_t* targets;          // may be null
    float tau;
    float *logp, *lse, *entropy;     // any may be null
    int top;
    int64_t* top_ids; float* top_logp;
    char* ws;
};
size_t logprob_workspace(int64_t k, int64_t batch, int64_t top);
hipError_t launch_logprob(const LogprobArgs& A, hipStream_t st);

struct LogprobBackwardArgs {
    const void* y;
    int64_t ldy, k, batch;
    bool bf16;
    const int64_t* targets;
    float tau;
    const float *lse, *entropy, *glogp, *gentropy, *glse;
    void* gy;
    int64_t ldgy;
};
hipError_t launch_logprob_backward(const LogprobBackwardArgs& A, hipStream_t st);

// ----------------------------------------------------------------------------
// Layer norm.
// ----------------------------------------------------------------------------
struct NormArgs {
    const void* x;
    void* y;
    int64_t ldx, ldy, rows, width;
    bool bf16;
    const float *weight, *bias;      // either may be null
    float eps;
    float *mean_out, *rstd_out;      // either may be null
};
hipError_t launch_norm(const NormArgs& A, hipStream_t st);

struct NormBackwardArgs {
    const void *x, *gy;
    void* gx;                        // may be null
    int64_t ldx, ldgy, ldgx, rows, width;
    bool bf16;
    const float *weight, *mean, *rstd;
    float *gweight, *gbias;          // either may be null
    float* parts;                    // [workgroups][2][width], null if neither is wanted
};
size_t norm_workspace(int64_t rows, int64_t width);
hipError_t launch_norm_backward(const NormBackwardArgs& A, hipStream_t st);

// ----------------------------------------------------------------------------
// Verification of drafted tokens.
// ----------------------------------------------------------------------------
enum { kVerifyNone, kVerifyPlace, kVerifyAll, kVerifyLeft, kVerifyOthers };      // the next token: none, the likeliest, from p, from max(p - q, 0), from p without the draft

struct VerifyColumn {
    double s, draft_s;               // sums of 2^(c (y - m)) of the two matrices
    int64_t place;                   // of the maximum, for the greedy rule
    float m, draft_m;
    int kept, mode;
};

struct VerifyArgs {
    const void *y, *z;               // z: the drafts' logits, or null
    int64_t ldy, ldz, k, batch, sequences;
    bool bf16, greedy;
    const int64_t *drafts, *starts;
    const double *chances, *next_chances;
    double tau, c, draft_c;          // c: tau / log 2
    int64_t *accepted, *next;
    float *logp, *next_logp;         // either may be null
    char* ws;
    // filled in by launch_verify
    int lanes_log2, seq_log2;
    int64_t part_rows, parts;
    double* part_sum; float* part_max; int64_t* part_place;      // [matrix][part][column]
    VerifyColumn* columns;
    double* left;                    // [part][sequence]
};
size_t verify_workspace(int64_t k, int64_t batch, int64_t sequences);
hipError_t launch_verify(const VerifyArgs& A, hipStream_t st);

#ifdef __HIPCC__
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__bf16 v) { return (float)v; }
#endif

}  // namespace laplex
