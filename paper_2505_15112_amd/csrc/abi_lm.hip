// abi_lm.hip -- the extern "C" entry points of the language model operators.
//
// As in abi.hip: arguments are checked on the host, before any HIP call, then
// the launchers of launch.hpp enqueue the kernels.
#include <limits.h>

#include "../../include/libscan.h"
#include "launch.hpp"

namespace {

constexpr int64_t kMaxBlocks = int64_t(1) << 23;  // of at most 512 threads each
constexpr int64_t kMaxSpan = int64_t(1) << 46;    // bytes from a tensor's first to its last

int64_t elem(int64_t type) { return type == LIBSCAN_F32 ? 4 : 2; }
bool known(int64_t type) {
    return type == LIBSCAN_F32 || type == LIBSCAN_F16 || type == LIBSCAN_BF16;
}

// The memory a tensor spans.  Inputs may be strided; nothing is read of a
// tensor without elements.
struct Span {
    const void* p;
    int64_t bytes;
    bool bad = false;
};
Span dense(const void* p, int64_t elems, int64_t es) { return {p, p ? elems * es : 0}; }
Span strided(const void* p, int64_t es, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2,
             int64_t s2, int64_t last) {
    if (n0 == 0 || n1 == 0 || n2 == 0 || last == 0) return {p, 0};
    if (s0 < 0 || s1 < 0 || s2 < 0) return {p, 0, true};
    const __int128 bytes =
        ((__int128)(n0 - 1) * s0 + (__int128)(n1 - 1) * s1 + (__int128)(n2 - 1) * s2 + last) * es;
    if (bytes > kMaxSpan) return {p, 0, true};
    return {p, (int64_t)bytes};
}

bool overlaps(const Span& a, const Span& b) {
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    return a.p && b.p && a.bytes && b.bytes && a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// Outputs clear of every input and of each other; inputs with sound strides.
template <int I, int O>
bool sound(const Span (&in)[I], const Span (&out)[O]) {
    for (int i = 0; i < I; ++i)
        if (in[i].bad) return false;
    for (int i = 0; i < O; ++i) {
        for (int j = 0; j < I; ++j)
            if (overlaps(out[i], in[j])) return false;
        for (int j = i + 1; j < O; ++j)
            if (overlaps(out[i], out[j])) return false;
    }
    return true;
}

int hip_status(hipError_t e) { return e == hipSuccess ? LIBSCAN_OK : LIBSCAN_EHIP; }

int check_scratch(const void* scratch, size_t bytes, size_t need) {
    if (need == 0) return LIBSCAN_OK;
    if (bytes < need) return LIBSCAN_ENOSPACE;
    return scratch && (uintptr_t)scratch % 16 == 0 ? LIBSCAN_OK : LIBSCAN_EINVAL;
}

// batch x steps x dim and what one launch and 32-bit indices inside a row hold
int check_sizes(int64_t batch, int64_t steps, int64_t dim) {
    if (batch < 0 || steps < 0 || dim < 0) return LIBSCAN_EINVAL;
    if (batch > kMaxBlocks || steps > INT32_MAX / 2 || dim > (1 << 24)) return LIBSCAN_ERANGE;
    if ((__int128)batch * (steps + 64) * (dim + 64) > ((__int128)1 << 42)) return LIBSCAN_ERANGE;
    return LIBSCAN_OK;
}

int check_conv(const libscan_conv* p) {
    if (!p || !known(p->type)) return LIBSCAN_EINVAL;
    if (p->weight_type != p->type && p->weight_type != LIBSCAN_F32) return LIBSCAN_EINVAL;
    if (p->width < 2 || p->width > 4) return LIBSCAN_EINVAL;
    const int r = check_sizes(p->batch, p->steps, p->dim);
    if (r != LIBSCAN_OK) return r;
    // forward threads own 8 steps of at least two channels, backward workgroups at
    // least 224 steps of 128
    if ((__int128)p->batch * (p->steps / 8 + 1) * (p->dim / 2 + 1) / 256 >= kMaxBlocks ||
        (__int128)p->batch * (p->steps / 224 + 1) * (p->dim / 128 + 1) >= kMaxBlocks)
        return LIBSCAN_ERANGE;
    return LIBSCAN_OK;
}

int64_t conv_window(const libscan_conv* p) { return p->batch * (p->width - 1) * p->dim; }

int check_ssm(const libscan_ssm* p) {
    if (!p || !known(p->type)) return LIBSCAN_EINVAL;
    if (p->n < 1 || p->groups < 1) return LIBSCAN_EINVAL;
    if (p->n > 64) return LIBSCAN_ERANGE;
    const int r = check_sizes(p->batch, p->steps, p->dim);
    if (r != LIBSCAN_OK) return r;
    if (p->dim % p->groups) return LIBSCAN_EINVAL;
    // workgroups of at least 16 channels, of 32 sums of dB, dC or dA, of 256 states
    const int64_t np = p->n <= 8 ? 8 : p->n <= 16 ? 16 : p->n <= 32 ? 32 : 64;
    if ((__int128)p->batch * p->groups * (p->dim / p->groups / 16 + 1) >= kMaxBlocks ||
        (__int128)p->batch * p->steps * p->groups * np / 32 >= kMaxBlocks ||
        (__int128)p->dim * np / 32 >= kMaxBlocks ||
        (__int128)p->batch * p->dim * np / 256 >= kMaxBlocks)
        return LIBSCAN_ERANGE;
    return LIBSCAN_OK;
}

// The spans of a scan's inputs; false if one that is needed is missing.
constexpr int kSsmInputs = 10;
bool ssm_inputs(const libscan_ssm* p, Span (&in)[kSsmInputs]) {
    const int64_t es = elem(p->type), b = p->batch, t = p->steps, d = p->dim, n = p->n;
    const int64_t tokens = b * t * d;
    if (tokens && (!p->x || !p->dt || !p->B || !p->C)) return false;
    if (d && !p->A) return false;
    in[0] = strided(p->x, es, b, p->x_batch, t, p->x_step, 1, 0, d);
    in[1] = strided(p->dt, es, b, p->dt_batch, t, p->dt_step, 1, 0, d);
    in[2] = p->z ? strided(p->z, es, b, p->z_batch, t, p->z_step, 1, 0, d) : Span{nullptr, 0};
    in[3] = strided(p->B, es, b, p->B_batch, t, p->B_step, p->groups, p->B_group, n);
    in[4] = strided(p->C, es, b, p->C_batch, t, p->C_step, p->groups, p->C_group, n);
    in[5] = dense(p->A, d * n, 4);
    in[6] = dense(p->D, d, 4);
    in[7] = dense(p->dt_bias, d, 4);
    in[8] = dense(p->state, b * d * n, 4);
    in[9] = dense(p->lengths, b, 4);
    return true;
}

int check_logits(const libscan_logits* p) {
    if (!p || !known(p->type) || p->rows < 0 || p->vocab < 0) return LIBSCAN_EINVAL;
    if (p->history_cols < 0 || p->biases < 0) return LIBSCAN_EINVAL;
    if (p->vocab > INT32_MAX - 65536 || p->history_cols > INT32_MAX - 65536 ||
        p->biases > INT32_MAX - 65536)
        return LIBSCAN_ERANGE;
    if (p->rows > kMaxBlocks || !ls::logits_fit(*p)) return LIBSCAN_ERANGE;
    return LIBSCAN_OK;
}

int check_attend(const libscan_attend* p) {
    if (!p || !known(p->type)) return LIBSCAN_EINVAL;
    if (p->dk < 1 || p->dv < 1 || p->heads < 0 || p->groups < 1) return LIBSCAN_EINVAL;
    // without heads there are groups all the same, and their gradients
    const int64_t most = p->heads ? p->heads : p->groups;
    if (p->dk > 256 || p->dv > 256 || most > (1 << 16)) return LIBSCAN_ERANGE;
    const int r = check_sizes(p->batch, p->steps, most * (p->dk > p->dv ? p->dk : p->dv));
    if (r != LIBSCAN_OK) return r;
    if (p->heads % p->groups) return LIBSCAN_EINVAL;
    // at most two workgroups to a row's head (more only where there are few)
    if ((__int128)p->batch * p->heads * 2 >= kMaxBlocks) return LIBSCAN_ERANGE;
    return LIBSCAN_OK;
}

// The spans of the attention's inputs; false if one that is needed is missing.
constexpr int kAttendInputs = 6;
bool attend_inputs(const libscan_attend* p, Span (&in)[kAttendInputs]) {
    const int64_t es = elem(p->type), b = p->batch, t = p->steps, h = p->heads, g = p->groups;
    if (b * t * h && (!p->q || !p->k || !p->v || !p->log_decay)) return false;
    in[0] = strided(p->q, es, b, p->q_batch, t, p->q_step, g, p->q_head, p->dk);
    in[1] = strided(p->k, es, b, p->k_batch, t, p->k_step, g, p->k_head, p->dk);
    in[2] = strided(p->v, es, b, p->v_batch, t, p->v_step, h, p->v_head, p->dv);
    in[3] = p->fixed ? dense(p->log_decay, h, 4)
                     : strided(p->log_decay, 4, b, p->decay_batch, t, p->decay_step, 1, 0, h);
    in[4] = dense(p->state, b * h * p->dk * p->dv, 4);
    in[5] = dense(p->lengths, b, 4);
    return true;
}

int check_norm(const libscan_norm* p) {
    if (!p || !known(p->type)) return LIBSCAN_EINVAL;
    if (p->weight_type != p->type && p->weight_type != LIBSCAN_F32) return LIBSCAN_EINVAL;
    if (p->groups < 1 || !(p->eps >= 0.0)) return LIBSCAN_EINVAL;
    const int r = check_sizes(p->batch, p->steps, p->dim);
    if (r != LIBSCAN_OK) return r;
    return p->dim % p->groups ? LIBSCAN_EINVAL : LIBSCAN_OK;
}

constexpr int kLogitsInputs = 11;
bool logits_inputs(const libscan_logits* p, Span (&in)[kLogitsInputs]) {
    const int64_t r = p->rows, v = p->vocab;
    if (r * v && !p->logits) return false;
    if (p->biases && (!p->bias_ids || !p->bias_values)) return false;
    in[0] = strided(p->logits, elem(p->type), r, p->logits_row, 1, 0, 1, 0, v);
    in[1] = p->history ? strided(p->history, 4, r, p->history_row, 1, 0, 1, 0, p->history_cols)
                       : Span{nullptr, 0};
    in[2] = dense(p->history_len, r, 4);
    in[3] = dense(p->prompt_len, r, 4);
    in[4] = dense(p->repetition, r, 4);
    in[5] = dense(p->presence, r, 4);
    in[6] = dense(p->frequency, r, 4);
    in[7] = dense(p->bias_ids, r * p->biases, 4);
    in[8] = dense(p->bias_values, r * p->biases, 4);
    in[9] = p->allowed ? strided(p->allowed, 4, r, p->allowed_row, 1, 0, 1, 0, (v + 31) / 32)
                       : Span{nullptr, 0};
    in[10] = dense(p->temperature, r, 4);
    return true;
}

}  // namespace

extern "C" {

int causal_conv(const libscan_conv* p, void* y, void* state_out, void* stream) {
    const int r = check_conv(p);
    if (r != LIBSCAN_OK) return r;
    const int64_t es = elem(p->type), tokens = p->batch * p->steps * p->dim;
    if ((tokens && (!p->x || !y)) || (p->batch * p->dim && !p->weight)) return LIBSCAN_EINVAL;
    const int64_t ws = elem(p->weight_type);
    const Span in[] = {strided(p->x, es, p->batch, p->x_batch, p->steps, p->x_step, 1, 0, p->dim),
                       dense(p->weight, p->dim * p->width, ws), dense(p->bias, p->dim, ws),
                       dense(p->state, conv_window(p), es), dense(p->lengths, p->batch, 4)};
    const Span out[] = {dense(y, tokens, es), dense(state_out, conv_window(p), es)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    return hip_status(ls::launch_conv(*p, y, state_out, (hipStream_t)stream));
}

int causal_conv_scratch_bytes(const libscan_conv* p, size_t* bytes) {
    const int r = check_conv(p);
    if (r != LIBSCAN_OK) return r;
    if (!bytes) return LIBSCAN_EINVAL;
    *bytes = ls::conv_scratch_bytes(*p);
    return LIBSCAN_OK;
}

int causal_conv_backward(const libscan_conv* p, const void* dy, int64_t dy_batch, int64_t dy_step,
                         const void* dstate_out, void* dx, float* dweight, float* dbias,
                         void* dstate, void* scratch, size_t scratch_bytes, void* stream) {
    const int r = check_conv(p);
    if (r != LIBSCAN_OK) return r;
    if (p->dim == 0) return LIBSCAN_OK;
    const int64_t es = elem(p->type), tokens = p->batch * p->steps * p->dim;
    if ((tokens && (!p->x || !dy || !dx)) || !p->weight || !dweight) return LIBSCAN_EINVAL;
    const int64_t ws = elem(p->weight_type);
    const size_t need = ls::conv_scratch_bytes(*p);
    const Span in[] = {strided(p->x, es, p->batch, p->x_batch, p->steps, p->x_step, 1, 0, p->dim),
                       dense(p->weight, p->dim * p->width, ws), dense(p->bias, p->dim, ws),
                       dense(p->state, conv_window(p), es), dense(p->lengths, p->batch, 4),
                       strided(dy, es, p->batch, dy_batch, p->steps, dy_step, 1, 0, p->dim),
                       dense(dstate_out, conv_window(p), es)};
    const Span out[] = {dense(dx, tokens, es), dense(dweight, p->dim * p->width, 4),
                        dense(dbias, p->dim, 4), dense(dstate, conv_window(p), es),
                        dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(ls::launch_conv_back(*p, dy, dy_batch, dy_step, dstate_out, dx, dweight,
                                           dbias, dstate, scratch, (hipStream_t)stream));
}

int causal_conv_step(const libscan_conv* p, void* states, int64_t n_states, const int32_t* slots,
                     void* y, void* stream) {
    const int r = check_conv(p);
    if (r != LIBSCAN_OK) return r;
    if (p->steps != 1 || p->state || p->lengths || n_states < 0) return LIBSCAN_EINVAL;
    if (p->batch == 0 || p->dim == 0) return LIBSCAN_OK;
    if (!p->x || !p->weight || !y || (n_states && !states)) return LIBSCAN_EINVAL;
    if (n_states > kMaxSpan / (p->dim * 16)) return LIBSCAN_ERANGE;
    const int64_t es = elem(p->type), ws = elem(p->weight_type);
    const Span in[] = {strided(p->x, es, p->batch, p->x_batch, 1, 0, 1, 0, p->dim),
                       dense(p->weight, p->dim * p->width, ws), dense(p->bias, p->dim, ws),
                       dense(slots, p->batch, 4)};
    const Span out[] = {dense(y, p->batch * p->dim, es),
                        dense(states, n_states * (p->width - 1) * p->dim, es)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    return hip_status(ls::launch_conv_step(*p, states, n_states, slots, y, (hipStream_t)stream));
}

int selective_scan_bytes(const libscan_ssm* p, size_t* checkpoints, size_t* scratch,
                         size_t* backward_scratch) {
    const int r = check_ssm(p);
    if (r != LIBSCAN_OK) return r;
    if (checkpoints) *checkpoints = ls::ssm_ckpt_bytes(*p);
    if (scratch) *scratch = ls::ssm_scratch_bytes(*p);
    if (backward_scratch) *backward_scratch = ls::ssm_back_scratch_bytes(*p);
    return LIBSCAN_OK;
}

int selective_scan(const libscan_ssm* p, void* y, float* state_out, float* checkpoints,
                   void* scratch, size_t scratch_bytes, void* stream) {
    const int r = check_ssm(p);
    if (r != LIBSCAN_OK) return r;
    const int64_t tokens = p->batch * p->steps * p->dim;
    Span in[kSsmInputs];
    if (!ssm_inputs(p, in) || (tokens && !y)) return LIBSCAN_EINVAL;
    const size_t need = ls::ssm_scratch_bytes(*p);
    const Span out[] = {dense(y, tokens, elem(p->type)),
                        dense(state_out, p->batch * p->dim * p->n, 4),
                        dense(checkpoints, (int64_t)ls::ssm_ckpt_bytes(*p), 1),
                        dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(
        ls::launch_ssm_scan(*p, y, state_out, checkpoints, scratch, (hipStream_t)stream));
}

int selective_scan_backward(const libscan_ssm* p, const void* dy, int64_t dy_batch,
                            int64_t dy_step, const float* checkpoints, const float* dstate_out,
                            void* dx, void* ddt, float* dA, void* dB, void* dC, float* dD,
                            void* dz, float* ddt_bias, float* dstate, void* scratch,
                            size_t scratch_bytes, void* stream) {
    const int r = check_ssm(p);
    if (r != LIBSCAN_OK) return r;
    const int64_t es = elem(p->type), tokens = p->batch * p->steps * p->dim;
    const int64_t states = p->batch * p->dim * p->n;
    const int64_t bc = p->batch * p->steps * p->groups * p->n;
    Span in[kSsmInputs + 3];
    Span(&first)[kSsmInputs] = (Span(&)[kSsmInputs])in;
    if (!ssm_inputs(p, first)) return LIBSCAN_EINVAL;
    if (tokens && (!dy || !checkpoints || !dx || !ddt || (p->z && !dz))) return LIBSCAN_EINVAL;
    if (bc && (!dB || !dC)) return LIBSCAN_EINVAL;
    if (p->dim && (!dA || (p->D && !dD) || (p->dt_bias && !ddt_bias))) return LIBSCAN_EINVAL;
    const size_t need = ls::ssm_back_scratch_bytes(*p);
    in[kSsmInputs] = strided(dy, es, p->batch, dy_batch, p->steps, dy_step, 1, 0, p->dim);
    in[kSsmInputs + 1] = dense(checkpoints, (int64_t)ls::ssm_ckpt_bytes(*p), 1);
    in[kSsmInputs + 2] = dense(dstate_out, states, 4);
    const Span out[] = {dense(dx, tokens, es),     dense(ddt, tokens, es), dense(dz, tokens, es),
                        dense(dA, p->dim * p->n, 4), dense(dB, bc, es),      dense(dC, bc, es),
                        dense(dD, p->dim, 4),      dense(ddt_bias, p->dim, 4),
                        dense(dstate, states, 4),  dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(ls::launch_ssm_back(*p, dy, dy_batch, dy_step, checkpoints, dstate_out, dx,
                                          ddt, dA, dB, dC, dD, dz, ddt_bias, dstate, scratch,
                                          (hipStream_t)stream));
}

int selective_scan_step(const libscan_ssm* p, float* states, int64_t n_states,
                        const int32_t* slots, void* y, void* stream) {
    const int r = check_ssm(p);
    if (r != LIBSCAN_OK) return r;
    if (p->steps != 1 || p->state || p->lengths || n_states < 0) return LIBSCAN_EINVAL;
    if (p->batch == 0 || p->dim == 0) return LIBSCAN_OK;
    Span in[kSsmInputs];
    if (!ssm_inputs(p, in) || !y || (n_states && !states)) return LIBSCAN_EINVAL;
    if (n_states > kMaxSpan / (p->dim * p->n * 4)) return LIBSCAN_ERANGE;
    in[8] = dense(slots, p->batch, 4);
    const Span out[] = {dense(y, p->batch * p->dim, elem(p->type)),
                        dense(states, n_states * p->dim * p->n, 4)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    return hip_status(ls::launch_ssm_step(*p, states, n_states, slots, y, (hipStream_t)stream));
}

int linear_attention_bytes(const libscan_attend* p, size_t* scratch, size_t* backward_scratch) {
    const int r = check_attend(p);
    if (r != LIBSCAN_OK) return r;
    if (scratch) *scratch = ls::attend_scratch_bytes(*p);
    if (backward_scratch) *backward_scratch = ls::attend_back_scratch_bytes(*p);
    return LIBSCAN_OK;
}

int linear_attention(const libscan_attend* p, void* y, float* state_out, void* scratch,
                     size_t scratch_bytes, void* stream) {
    const int r = check_attend(p);
    if (r != LIBSCAN_OK) return r;
    const int64_t values = p->batch * p->steps * p->heads * p->dv;
    Span in[kAttendInputs];
    if (!attend_inputs(p, in) || (values && !y)) return LIBSCAN_EINVAL;
    const size_t need = ls::attend_scratch_bytes(*p);
    const Span out[] = {dense(y, values, elem(p->type)),
                        dense(state_out, p->batch * p->heads * p->dk * p->dv, 4),
                        dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(ls::launch_attend(*p, y, state_out, scratch, (hipStream_t)stream));
}

int linear_attention_backward(const libscan_attend* p, const void* dy, int64_t dy_batch,
                              int64_t dy_step, int64_t dy_head, const float* dstate_out, void* dq,
                              void* dk, void* dv, float* dlog_decay, float* dstate, void* scratch,
                              size_t scratch_bytes, void* stream) {
    const int r = check_attend(p);
    if (r != LIBSCAN_OK) return r;
    const int64_t es = elem(p->type), b = p->batch, t = p->steps, h = p->heads;
    const int64_t states = b * h * p->dk * p->dv, shared = b * t * p->groups * p->dk;
    Span in[kAttendInputs + 2];
    Span(&first)[kAttendInputs] = (Span(&)[kAttendInputs])in;
    if (!attend_inputs(p, first)) return LIBSCAN_EINVAL;
    if ((b * t * h && (!dy || !dv)) || (shared && (!dq || !dk))) return LIBSCAN_EINVAL;
    if ((p->fixed ? h : b * t * h) && !dlog_decay) return LIBSCAN_EINVAL;
    const size_t need = ls::attend_back_scratch_bytes(*p);
    in[kAttendInputs] = strided(dy, es, b, dy_batch, t, dy_step, h, dy_head, p->dv);
    in[kAttendInputs + 1] = dense(dstate_out, states, 4);
    const Span out[] = {dense(dq, shared, es), dense(dk, shared, es),
                        dense(dv, b * t * h * p->dv, es),
                        dense(dlog_decay, p->fixed ? h : b * t * h, 4), dense(dstate, states, 4),
                        dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(ls::launch_attend_back(*p, dy, dy_batch, dy_step, dy_head, dstate_out, dq, dk,
                                             dv, dlog_decay, dstate, scratch,
                                             (hipStream_t)stream));
}

int linear_attention_step(const libscan_attend* p, float* states, int64_t n_states,
                          const int32_t* slots, void* y, void* stream) {
    const int r = check_attend(p);
    if (r != LIBSCAN_OK) return r;
    if (p->steps != 1 || p->state || p->lengths || n_states < 0) return LIBSCAN_EINVAL;
    if (p->batch == 0 || p->heads == 0) return LIBSCAN_OK;
    Span in[kAttendInputs];
    if (!attend_inputs(p, in) || !y || (n_states && !states)) return LIBSCAN_EINVAL;
    const int64_t each = p->heads * p->dk * p->dv;
    if (n_states > kMaxSpan / (each * 4)) return LIBSCAN_ERANGE;
    in[4] = dense(slots, p->batch, 4);
    const Span out[] = {dense(y, p->batch * p->heads * p->dv, elem(p->type)),
                        dense(states, n_states * each, 4)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    return hip_status(ls::launch_attend_step(*p, states, n_states, slots, y, (hipStream_t)stream));
}

int layer_norm(const libscan_norm* p, void* y, void* sum, float* stats, void* stream) {
    const int r = check_norm(p);
    if (r != LIBSCAN_OK) return r;
    const int64_t es = elem(p->type), ws = elem(p->weight_type), rows = p->batch * p->steps;
    if (rows * p->dim && (!p->x || !y)) return LIBSCAN_EINVAL;
    const Span in[] = {strided(p->x, es, p->batch, p->x_batch, p->steps, p->x_step, 1, 0, p->dim),
                       p->residual ? strided(p->residual, es, p->batch, p->residual_batch, p->steps,
                                             p->residual_step, 1, 0, p->dim)
                                   : Span{nullptr, 0},
                       dense(p->weight, p->dim, ws), dense(p->bias, p->dim, ws)};
    const Span out[] = {dense(y, rows * p->dim, es), dense(sum, rows * p->dim, es),
                        dense(stats, rows * p->groups * 2, 4)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    return hip_status(ls::launch_norm(*p, y, sum, stats, (hipStream_t)stream));
}

int layer_norm_scratch_bytes(const libscan_norm* p, size_t* bytes) {
    const int r = check_norm(p);
    if (r != LIBSCAN_OK) return r;
    if (!bytes) return LIBSCAN_EINVAL;
    *bytes = ls::norm_scratch_bytes(*p);
    return LIBSCAN_OK;
}

int layer_norm_backward(const libscan_norm* p, const void* dy, int64_t dy_batch, int64_t dy_step,
                        const void* dsum, int64_t dsum_batch, int64_t dsum_step,
                        const float* stats, void* dx, float* dweight, float* dbias, void* scratch,
                        size_t scratch_bytes, void* stream) {
    const int r = check_norm(p);
    if (r != LIBSCAN_OK) return r;
    if (p->residual) return LIBSCAN_EINVAL;
    const int64_t es = elem(p->type), ws = elem(p->weight_type), rows = p->batch * p->steps;
    if (rows * p->dim && (!p->x || !dy || !stats || !dx)) return LIBSCAN_EINVAL;
    const size_t need = ls::norm_scratch_bytes(*p);
    const Span in[] = {strided(p->x, es, p->batch, p->x_batch, p->steps, p->x_step, 1, 0, p->dim),
                       strided(dy, es, p->batch, dy_batch, p->steps, dy_step, 1, 0, p->dim),
                       dsum ? strided(dsum, es, p->batch, dsum_batch, p->steps, dsum_step, 1, 0,
                                      p->dim)
                            : Span{nullptr, 0},
                       dense(p->weight, p->dim, ws), dense(p->bias, p->dim, ws),
                       dense(stats, rows * p->groups * 2, 4)};
    const Span out[] = {dense(dx, rows * p->dim, es), dense(dweight, p->dim, 4),
                        dense(dbias, p->dim, 4), dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(ls::launch_norm_back(*p, dy, dy_batch, dy_step, dsum, dsum_batch, dsum_step,
                                           stats, dx, dweight, dbias, scratch,
                                           (hipStream_t)stream));
}

int logits_process(const libscan_logits* p, void* out, int64_t out_row, void* stream) {
    const int r = check_logits(p);
    if (r != LIBSCAN_OK) return r;
    Span in[kLogitsInputs];
    if (!logits_inputs(p, in)) return LIBSCAN_EINVAL;
    if (p->rows * p->vocab == 0) return LIBSCAN_OK;
    if (!out || (p->rows > 1 && out_row < p->vocab)) return LIBSCAN_EINVAL;
    const Span o[] = {strided(out, elem(p->type), p->rows, out_row, 1, 0, 1, 0, p->vocab)};
    if (o[0].bad) return LIBSCAN_EINVAL;
    // in place: every place is read and written by one thread
    if (out == p->logits && (out_row == p->logits_row || p->rows == 1)) in[0].bytes = 0;
    if (!sound(in, o)) return LIBSCAN_EINVAL;
    return hip_status(ls::launch_logits_process(*p, out, out_row, (hipStream_t)stream));
}

int logits_scratch_bytes(const libscan_logits* p, size_t* bytes) {
    const int r = check_logits(p);
    if (r != LIBSCAN_OK) return r;
    if (!bytes) return LIBSCAN_EINVAL;
    *bytes = ls::logits_scratch(*p);
    return LIBSCAN_OK;
}

int logits_probs(const libscan_logits* p, float* probs, void* scratch, size_t scratch_bytes,
                 void* stream) {
    const int r = check_logits(p);
    if (r != LIBSCAN_OK) return r;
    Span in[kLogitsInputs];
    if (!logits_inputs(p, in)) return LIBSCAN_EINVAL;
    if (p->rows * p->vocab == 0) return LIBSCAN_OK;
    if (!probs) return LIBSCAN_EINVAL;
    const size_t need = ls::logits_scratch(*p);
    const Span out[] = {dense(probs, p->rows * p->vocab, 4), dense(scratch, (int64_t)need, 1)};
    if (!sound(in, out)) return LIBSCAN_EINVAL;
    const int s = check_scratch(scratch, scratch_bytes, need);
    if (s != LIBSCAN_OK) return s;
    return hip_status(ls::launch_logits_probs(*p, probs, scratch, (hipStream_t)stream));
}

}  // extern "C"
