// Host side of the operators for token models: argument checks (before any HIP call) and the kernels' arguments.
#include "../../include/laplex.h"
#include "token_internal.h"

#include <cmath>

using namespace laplex;

namespace {

#define LAPLEX_CHECK(expr)                       \
    do {                                         \
        const int rc_ = (expr);                  \
        if (rc_ != LAPLEX_OK) return rc_;        \
    } while (0)

#define LAPLEX_HIP(expr)                                   \
    do {                                                   \
        const hipError_t e_ = (expr);                      \
        if (e_ != hipSuccess) return hip_failed(e_);       \
    } while (0)

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int check_type(int type) { return type == LAPLEX_F32 || type == LAPLEX_BF16 ? LAPLEX_OK : LAPLEX_ERR_VALUE; }

int64_t bytes_of(int type) { return type == LAPLEX_BF16 ? 2 : 4; }

// a matrix of `rows` rows of `width` elements that lie ld apart
int check_rows(const void* p, int type, int64_t rows, int64_t width, int64_t ld, bool required)
{
    if (rows == 0 || width == 0) return LAPLEX_OK;     // never dereferenced
    if (!p) return required ? LAPLEX_ERR_NULL : LAPLEX_OK;
    if (misaligned(p, (uintptr_t)bytes_of(type))) return LAPLEX_ERR_ALIGN;
    if (ld < width) return LAPLEX_ERR_LD;
    return rows > (INT64_MAX / 8) / ld ? LAPLEX_ERR_SIZE : LAPLEX_OK;
}

int check_array(const void* p, int64_t length, uintptr_t align, bool required)
{
    if (length == 0) return LAPLEX_OK;
    if (!p) return required ? LAPLEX_ERR_NULL : LAPLEX_OK;
    return misaligned(p, align) ? LAPLEX_ERR_ALIGN : LAPLEX_OK;
}

int check_ws(const void* ws, size_t have, size_t need)
{
    if (need == 0) return LAPLEX_OK;
    if (!ws) return LAPLEX_ERR_NULL;
    if (misaligned(ws, 256)) return LAPLEX_ERR_ALIGN;
    return have < need ? LAPLEX_ERR_WORKSPACE : LAPLEX_OK;
}

int check_attention_sizes(int type, int64_t tokens, int64_t sequences, int64_t heads, int64_t dk, int64_t dv, bool equal)
{
    LAPLEX_CHECK(check_type(type));
    if (tokens < 0 || sequences < 0 || heads < 0 || heads > LAPLEX_TOKEN_MAX_HEADS) return LAPLEX_ERR_SIZE;
    if (dk < 1 || dv < 1 || dk > LAPLEX_ATTENTION_MAX_DIM || dv > LAPLEX_ATTENTION_MAX_DIM) return LAPLEX_ERR_SIZE;
    if (tokens > LAPLEX_TOKEN_MAX_TOKENS || sequences > LAPLEX_TOKEN_MAX_SEQUENCES) return LAPLEX_ERR_SIZE;
    if (equal && (sequences == 0 ? tokens != 0 : tokens % sequences != 0)) return LAPLEX_ERR_SIZE;
    return LAPLEX_OK;
}

bool positive(float v) { return v > 0.0f && std::isfinite(v); }

}  // namespace

extern "C" {

int laplex_rotary(const void* x, int64_t ldx, void* y, int64_t ldy, int type, int64_t tokens, int64_t heads, int64_t head_dim,
                  int64_t rotary_dim, const int64_t* positions, const float* frequencies, float magnitude, uint32_t flags,
                  laplex_stream_t stream)
{
    LAPLEX_CHECK(check_type(type));
    if (flags & ~(LAPLEX_ROTARY_INTERLEAVED | LAPLEX_ROTARY_INVERSE)) return LAPLEX_ERR_FLAGS;
    if (tokens < 0 || tokens > LAPLEX_TOKEN_MAX_TOKENS || heads < 0 || heads > LAPLEX_TOKEN_MAX_HEADS) return LAPLEX_ERR_SIZE;
    if (head_dim < 0 || head_dim > LAPLEX_ROTARY_MAX_DIM || rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 2 != 0)
        return LAPLEX_ERR_SIZE;
    if (!std::isfinite(magnitude)) return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_rows(x, type, tokens, heads * head_dim, ldx, true));
    LAPLEX_CHECK(check_rows(y, type, tokens, heads * head_dim, ldy, true));
    if (tokens == 0 || heads == 0 || head_dim == 0) return LAPLEX_OK;
    LAPLEX_CHECK(check_array(positions, rotary_dim, 8, true));
    LAPLEX_CHECK(check_array(frequencies, rotary_dim, 4, true));
    RotaryArgs A{};
    A.x = x; A.y = y; A.ldx = ldx; A.ldy = ldy; A.tokens = tokens;
    A.heads = (int)heads; A.dim = (int)head_dim; A.half = (int)(rotary_dim / 2);
    A.positions = positions; A.frequencies = frequencies; A.magnitude = magnitude;
    A.bf16 = type == LAPLEX_BF16;
    A.interleaved = (flags & LAPLEX_ROTARY_INTERLEAVED) != 0; A.inverse = (flags & LAPLEX_ROTARY_INVERSE) != 0;
    LAPLEX_HIP(launch_rotary(A, stream));
    return LAPLEX_OK;
}

int laplex_rotary_frequencies(float* frequencies, int64_t rotary_dim, double base, int scaling, double factor,
                              double original_context, double low_turns, double high_turns, laplex_stream_t stream)
{
    if (rotary_dim < 0 || rotary_dim > LAPLEX_ROTARY_MAX_DIM || rotary_dim % 2 != 0) return LAPLEX_ERR_SIZE;
    if (scaling < LAPLEX_ROTARY_PLAIN || scaling > LAPLEX_ROTARY_PARTS) return LAPLEX_ERR_VALUE;
    if (!(base > 0.0) || !std::isfinite(base)) return LAPLEX_ERR_VALUE;
    if (scaling != LAPLEX_ROTARY_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return LAPLEX_ERR_VALUE;
    if (scaling == LAPLEX_ROTARY_PARTS && (!(original_context > 0.0) || !std::isfinite(original_context) ||
                                           !std::isfinite(low_turns) || !std::isfinite(high_turns) || !(low_turns < high_turns)))
        return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_array(frequencies, rotary_dim, 4, true));
    if (rotary_dim == 0) return LAPLEX_OK;
    LAPLEX_HIP(launch_rotary_frequencies(frequencies, rotary_dim / 2, base, scaling, factor, original_context, low_turns, high_turns, stream));
    return LAPLEX_OK;
}

int laplex_decay_attention_workspace_bytes(int type, int64_t tokens, int64_t sequences, int64_t heads, int64_t dk, int64_t dv, size_t* out)
{
    if (!out) return LAPLEX_ERR_NULL;
    LAPLEX_CHECK(check_attention_sizes(type, tokens, sequences, heads, dk, dv, false));
    *out = attention_workspace(tokens, sequences, (int)heads, (int)dk, (int)dv);
    return LAPLEX_OK;
}

int laplex_decay_attention(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int type,
                           int64_t tokens, int64_t sequences, const int64_t* starts, int64_t heads, int64_t dk, int64_t dv,
                           const float* rates, float scale, const float* state_in, void* y, int64_t ldy, float* state_out,
                           void* ws, size_t ws_bytes, laplex_stream_t stream)
{
    LAPLEX_CHECK(check_attention_sizes(type, tokens, sequences, heads, dk, dv, starts == nullptr));
    if (!positive(scale)) return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_rows(q, type, tokens, heads * dk, ldq, true));
    LAPLEX_CHECK(check_rows(k, type, tokens, heads * dk, ldk, true));
    LAPLEX_CHECK(check_rows(v, type, tokens, heads * dv, ldv, true));
    LAPLEX_CHECK(check_rows(y, type, tokens, heads * dv, ldy, true));
    LAPLEX_CHECK(check_array(starts, sequences, 8, false));
    LAPLEX_CHECK(check_array(rates, heads, 4, true));
    LAPLEX_CHECK(check_array(state_in, sequences * heads, 4, false));
    LAPLEX_CHECK(check_array(state_out, sequences * heads, 4, false));
    if (sequences == 0 || heads == 0 || (tokens == 0 && !state_out)) return LAPLEX_OK;
    LAPLEX_CHECK(check_ws(ws, ws_bytes, attention_workspace(tokens, sequences, (int)heads, (int)dk, (int)dv)));
    AttentionArgs A{};
    A.starts = starts; A.tokens = tokens; A.sequences = sequences; A.heads = (int)heads; A.rates = rates;
    A.bf16 = type == LAPLEX_BF16; A.ws = static_cast<char*>(ws);
    Walk& W = A.walk[A.walks++];
    W.q = q; W.ldq = ldq; W.k = k; W.ldk = ldk; W.v = v; W.ldv = ldv; W.out = y; W.ldo = ldy;
    W.dk = (int)dk; W.dv = (int)dv; W.lead = 1; W.exact = 1;
    W.state_in = state_in; W.inner = W.last_scale = 1.0f;
    W.state_out = state_out;
    W.out_scale = scale;
    A.states[A.sets++] = W;
    LAPLEX_HIP(launch_attention(A, stream));
    return LAPLEX_OK;
}

int laplex_decay_attention_backward(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int type,
                                    int64_t tokens, int64_t sequences, const int64_t* starts, int64_t heads, int64_t dk, int64_t dv,
                                    const float* rates, float scale, const float* state_in, const void* gy, int64_t ldgy,
                                    const float* gstate_out, void* gq, int64_t ldgq, void* gk, int64_t ldgk, void* gv, int64_t ldgv,
                                    float* gstate_in, void* ws, size_t ws_bytes, laplex_stream_t stream)
{
    LAPLEX_CHECK(check_attention_sizes(type, tokens, sequences, heads, dk, dv, starts == nullptr));
    if (!positive(scale)) return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_rows(q, type, tokens, heads * dk, ldq, true));
    LAPLEX_CHECK(check_rows(k, type, tokens, heads * dk, ldk, true));
    LAPLEX_CHECK(check_rows(v, type, tokens, heads * dv, ldv, true));
    LAPLEX_CHECK(check_rows(gy, type, tokens, heads * dv, ldgy, true));
    LAPLEX_CHECK(check_rows(gq, type, tokens, heads * dk, ldgq, false));
    LAPLEX_CHECK(check_rows(gk, type, tokens, heads * dk, ldgk, false));
    LAPLEX_CHECK(check_rows(gv, type, tokens, heads * dv, ldgv, false));
    LAPLEX_CHECK(check_array(starts, sequences, 8, false));
    LAPLEX_CHECK(check_array(rates, heads, 4, true));
    LAPLEX_CHECK(check_array(state_in, sequences * heads, 4, false));
    LAPLEX_CHECK(check_array(gstate_out, sequences * heads, 4, false));
    LAPLEX_CHECK(check_array(gstate_in, sequences * heads, 4, false));
    if (sequences == 0 || heads == 0 || (tokens == 0 && !gstate_in) || (!gq && !gk && !gv && !gstate_in)) return LAPLEX_OK;
    LAPLEX_CHECK(check_ws(ws, ws_bytes, attention_workspace(tokens, sequences, (int)heads, (int)dk, (int)dv)));
    AttentionArgs A{};
    A.starts = starts; A.tokens = tokens; A.sequences = sequences; A.heads = (int)heads; A.rates = rates;
    A.bf16 = type == LAPLEX_BF16; A.ws = static_cast<char*>(ws);
    A.backward = true;
    // The walks back weight their sums by the scale, but not the state they begin from: the scale goes into the sums, as far as it leaves their parts room, and what is
    // left of it around them (gstate_out / scale alone would overflow where neither it nor the gradients do).
    const float inner = scale < 0x1p-40f ? 0x1p-40f : scale > 0x1p40f ? 0x1p40f : scale, outer = scale / inner;
    // back: queries k, keys q, values gy.  The states of both walks back are these, whichever of the two is wanted, so that neither depends on the other.
    Walk B{};
    B.q = k; B.ldq = ldk; B.k = q; B.ldk = ldq; B.v = gy; B.ldv = ldgy; B.out = gv; B.ldo = ldgv;
    B.dk = (int)dk; B.dv = (int)dv; B.reverse = 1; B.exact = 1;
    B.state_in = gstate_out; B.inner = inner; B.out_scale = outer;
    B.state_out = gstate_in; B.last_scale = outer;
    B.set = A.sets;
    if (gk || gv || gstate_in) A.states[A.sets++] = B;
    if (gk) {        // back: queries v, keys gy, values q, the transposed state
        Walk& W = A.walk[A.walks++];
        W.set = B.set; W.set_transposed = 1;
        W.q = v; W.ldq = ldv; W.k = gy; W.ldk = ldgy; W.v = q; W.ldv = ldq; W.out = gk; W.ldo = ldgk;
        W.dk = (int)dv; W.dv = (int)dk; W.reverse = 1; W.transposed = 1;
        W.state_in = gstate_out; W.inner = inner; W.out_scale = W.last_scale = outer;
    }
    if (gv || gstate_in) A.walk[A.walks++] = B;
    if (gq) {        // ahead: queries gy, keys v, values k, the transposed state
        Walk& W = A.walk[A.walks++];
        W.q = gy; W.ldq = ldgy; W.k = v; W.ldk = ldv; W.v = k; W.ldv = ldk; W.out = gq; W.ldo = ldgq;
        W.dk = (int)dv; W.dv = (int)dk; W.lead = 1; W.transposed = 1;
        W.state_in = state_in; W.inner = W.last_scale = 1.0f; W.out_scale = scale;
        W.set = A.sets;
        A.states[A.sets++] = W;
    }
    LAPLEX_HIP(launch_attention(A, stream));
    return LAPLEX_OK;
}

int laplex_decay_attention_step(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int type,
                                int64_t sequences, int64_t heads, int64_t dk, int64_t dv, const float* rates, float scale,
                                float* state, void* y, int64_t ldy, laplex_stream_t stream)
{
    LAPLEX_CHECK(check_attention_sizes(type, sequences, sequences, heads, dk, dv, true));
    if (!positive(scale)) return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_rows(q, type, sequences, heads * dk, ldq, true));
    LAPLEX_CHECK(check_rows(k, type, sequences, heads * dk, ldk, true));
    LAPLEX_CHECK(check_rows(v, type, sequences, heads * dv, ldv, true));
    LAPLEX_CHECK(check_rows(y, type, sequences, heads * dv, ldy, true));
    LAPLEX_CHECK(check_array(rates, heads, 4, true));
    LAPLEX_CHECK(check_array(state, sequences * heads, 4, true));
    if (sequences == 0 || heads == 0) return LAPLEX_OK;
    AttentionStepArgs A{};
    A.q = q; A.k = k; A.v = v; A.y = y; A.ldq = ldq; A.ldk = ldk; A.ldv = ldv; A.ldy = ldy; A.sequences = sequences;
    A.heads = (int)heads; A.dk = (int)dk; A.dv = (int)dv; A.rates = rates; A.scale = scale; A.state = state;
    A.bf16 = type == LAPLEX_BF16;
    LAPLEX_HIP(launch_attention_step(A, stream));
    return LAPLEX_OK;
}

int laplex_logprob_workspace_bytes(int64_t k, int64_t batch, int64_t top, size_t* out)
{
    if (!out) return LAPLEX_ERR_NULL;
    if (k < 0 || batch < 0 || k > kLogprobMaxRows || batch > LAPLEX_TOKEN_MAX_TOKENS || top < 0 || top > LAPLEX_LOGPROB_MAX_TOP || top > k)
        return LAPLEX_ERR_SIZE;
    *out = logprob_workspace(k, batch, top);
    return LAPLEX_OK;
}

int laplex_logprob(const void* y, int64_t ldy, int type, int64_t k, int64_t batch, const int64_t* targets, float tau,
                   float* logp, float* lse, float* entropy, int64_t top, int64_t* top_ids, float* top_logp,
                   void* ws, size_t ws_bytes, laplex_stream_t stream)
{
    LAPLEX_CHECK(check_type(type));
    size_t need = 0;
    LAPLEX_CHECK(laplex_logprob_workspace_bytes(k, batch, top, &need));
    if (!positive(tau)) return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_rows(y, type, k, batch, ldy, true));
    LAPLEX_CHECK(check_array(targets, batch, 8, logp != nullptr));
    LAPLEX_CHECK(check_array(logp, batch, 4, false));
    LAPLEX_CHECK(check_array(lse, batch, 4, false));
    LAPLEX_CHECK(check_array(entropy, batch, 4, false));
    LAPLEX_CHECK(check_array(top_ids, top * batch, 8, true));
    LAPLEX_CHECK(check_array(top_logp, top * batch, 4, true));
    if (batch == 0 || (!logp && !lse && !entropy && top == 0)) return LAPLEX_OK;
    LAPLEX_CHECK(check_ws(ws, ws_bytes, need));
    LogprobArgs A{};
    A.y = y; A.ldy = ldy; A.k = k; A.batch = batch; A.bf16 = type == LAPLEX_BF16; A.targets = targets; A.tau = tau;
    A.logp = logp; A.lse = lse; A.entropy = entropy; A.top = (int)top; A.top_ids = top_ids; A.top_logp = top_logp;
    A.ws = static_cast<char*>(ws);
    LAPLEX_HIP(launch_logprob(A, stream));
    return LAPLEX_OK;
}

int laplex_logprob_backward(const void* y, int64_t ldy, int type, int64_t k, int64_t batch, const int64_t* targets, float tau,
                            const float* lse, const float* entropy, const float* glogp, const float* gentropy, const float* glse,
                            void* gy, int64_t ldgy, laplex_stream_t stream)
{
    LAPLEX_CHECK(check_type(type));
    if (k < 0 || batch < 0 || k > kLogprobMaxRows || batch > LAPLEX_TOKEN_MAX_TOKENS) return LAPLEX_ERR_SIZE;
    if (!positive(tau)) return LAPLEX_ERR_VALUE;
    LAPLEX_CHECK(check_rows(y, type, k, batch, ldy, true));
    LAPLEX_CHECK(check_rows(gy, type, k, batch, ldgy, true));
    LAPLEX_CHECK(check_array(targets, batch, 8, glogp != nullptr));
    LAPLEX_CHECK(check_array(lse, batch, 4, true));
    LAPLEX_CHECK(check_array(entropy, batch, 4, gentropy != nullptr));
    LAPLEX_CHECK(check_array(glogp, batch, 4, false));
    LAPLEX_CHECK(check_array(gentropy, batch, 4, false));
    LAPLEX_CHECK(check_array(glse, batch, 4, false));
    if (k == 0 || batch == 0) return LAPLEX_OK;
    LogprobBackwardArgs A{};
    A.y = y; A.ldy = ldy; A.k = k; A.batch = batch; A.bf16 = type == LAPLEX_BF16; A.targets = targets; A.tau = tau;
    A.lse = lse; A.entropy = entropy; A.glogp = glogp; A.gentropy = gentropy; A.glse = glse; A.gy = gy; A.ldgy = ldgy;
    LAPLEX_HIP(launch_logprob_backward(A, stream));
    return LAPLEX_OK;
}

}  // extern "C"
