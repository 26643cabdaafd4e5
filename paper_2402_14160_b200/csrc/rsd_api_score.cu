// C ABI of librsd (declared in include/rsd.h), scoring part: argument checks and kernel launches, nothing else.
#include <algorithm>
#include <cstring>

#include "rsd_api_common.h"
#include "rsd_score_args.h"

using namespace rsd_host;

namespace {

int check_entries(const char* name, const rsd_rows* r) {   // entries on their own boundaries: a row is read in granules around it
    if ((uintptr_t)r->data % (r->dtype == RSD_F32 ? 4 : 2)) return fail(RSD_ERR_INVALID_ARG, "%s: not on an element boundary", name);
    return RSD_OK;
}
int check_batch(int B, int R) {
    if (B < 0 || R < 1) return fail(RSD_ERR_INVALID_ARG, "B = %d, R = %d", B, R);
    if ((int64_t)B * R > 0x7FFFFFFF) return fail(RSD_ERR_UNSUPPORTED, "B * R too large");
    return RSD_OK;
}
// Whether `bytes` from `out` on lie over an entry of the rows [B][R][V]; memory between the rows is not theirs.
bool over_rows(const rsd_rows* rows, int B, int R, int V, const void* out, int64_t bytes) {
    typedef __int128 wide;                                       // (strides may be anything that 64 bits hold)
    const int64_t elem = rows->dtype == RSD_F32 ? 4 : 2;
    const wide lo = (wide)(uintptr_t)out - (wide)(uintptr_t)rows->data, hi = lo + bytes, row = (wide)V * elem;
    const wide row_step = (wide)rows->row_stride * elem, seq_step = (wide)rows->seq_stride * elem;
    const wide sequence = row_step * (R - 1) + row;              // from a sequence's first entry to behind its last
    // of pieces of `length` bytes, one every `step` bytes, the first that ends behind `from`
    const auto first = [](wide step, wide length, wide from) { return from < length || step == 0 ? (wide)0 : (from - length) / step + 1; };
    for (wide b = first(seq_step, sequence, lo); b < B && b * seq_step < hi; ++b) {
        const wide start = b * seq_step, r = first(row_step, row, lo - start), at = start + r * row_step;
        if (r < R && at < hi && at + row > lo) return true;
        if (seq_step == 0) break;
    }
    return false;
}
float inverse(float temp) { return (float)std::min(1.0 / (double)temp, 3.0e38); }
float exponent_scale(float temp) { return (float)std::min(1.4426950408889634 / (double)temp, 3.0e38); }   // log2(e) / T
bool dense_aligned(const void* p, int V, int dtype) { return (uintptr_t)p % 16 == 0 && (int64_t)V * (dtype == RSD_F32 ? 4 : 2) % 16 == 0; }

rsd::ScoreArgs score_args(const rsd_rows* rows, int R, int V, int T, int K) {
    rsd::ScoreArgs a;
    memset(&a, 0, sizeof(a));
    a.data = rows->data; a.seq_stride = rows->seq_stride; a.row_stride = rows->row_stride;
    a.R = R; a.V = V; a.T = T; a.K = K;
    const float temp = temperature_of(rows);
    a.inv_temp = inverse(temp); a.k = exponent_scale(temp);
    return a;
}
rsd::DivergenceArgs divergence_args(const rsd_rows* draft, const rsd_rows* target, int R, int V) {
    rsd::DivergenceArgs a;
    memset(&a, 0, sizeof(a));
    a.draft = draft->data; a.draft_seq = draft->seq_stride; a.draft_row = draft->row_stride;
    a.target = target->data; a.target_seq = target->seq_stride; a.target_row = target->row_stride;
    a.R = R; a.V = V;
    a.inv_draft_temp = inverse(temperature_of(draft));
    a.k_draft = exponent_scale(temperature_of(draft)); a.k_target = exponent_scale(temperature_of(target));
    return a;
}
int check_pair(const rsd_rows* draft, const rsd_rows* target, int B, int R, int V) {
    if (int e = check_vocab(V)) return e;
    if (int e = check_rows("draft", draft, V, R > 1)) return e;
    if (int e = check_rows("target", target, V, R > 1)) return e;
    if (int e = check_entries("draft", draft)) return e;
    if (int e = check_entries("target", target)) return e;
    if (draft->dtype != target->dtype) return fail(RSD_ERR_UNSUPPORTED, "draft and target rows must have the same dtype");
    return check_batch(B, R);
}

int launch_scores(const rsd_rows* rows, int B, const rsd::ScoreArgs& a, cudaStream_t s, const char* what) {
    const unsigned slots = (unsigned)((int64_t)B * a.R);
    if (rows->dtype == RSD_F32) rsd::launch_score_f32(rows_aligned(rows), slots, a, s);
    else rsd::launch_score_bf16(rows_aligned(rows), slots, a, s);
    return check_launch(what);
}

}  // namespace

extern "C" {

int rsd_token_logprobs(const rsd_rows* rows, int B, int R, int V, int num_rows, const int32_t* row_index, const int32_t* token, int T,
                       int K, float* out_logprob, float* out_entropy, int32_t* out_top_token, float* out_top_logprob,
                       int32_t* status, rsd_stream_t stream) {
    g_err[0] = 0;
    if (int e = check_vocab(V)) return e;
    if (num_rows < 1) return fail(RSD_ERR_INVALID_ARG, "num_rows = %d", num_rows);
    if (int e = check_rows("rows", rows, V, num_rows > 1)) return e;
    if (int e = check_entries("rows", rows)) return e;
    if (int e = check_batch(B, R)) return e;
    if (!row_index && R > num_rows) return fail(RSD_ERR_INVALID_ARG, "R = %d > num_rows = %d without a row_index", R, num_rows);
    if (T < 0 || T > RSD_MAX_K) return fail(RSD_ERR_UNSUPPORTED, "T = %d outside [0, %d]", T, (int)RSD_MAX_K);
    if (K < 0 || K > RSD_MAX_K) return fail(RSD_ERR_UNSUPPORTED, "K = %d outside [0, %d]", K, (int)RSD_MAX_K);
    if (!status || (T > 0 && (!token || !out_logprob)) || (K > 0 && (!out_top_token || !out_top_logprob))) return fail(RSD_ERR_INVALID_ARG, "null argument");
    if (B == 0) return RSD_OK;
    rsd::ScoreArgs a = score_args(rows, R, V, T, K);
    a.num_rows = num_rows; a.row_index = row_index; a.token = token;
    a.out_logprob = out_logprob; a.out_entropy = out_entropy; a.out_top_token = out_top_token; a.out_top_logprob = out_top_logprob;
    a.status = status;
    return launch_scores(rows, B, a, (cudaStream_t)stream, "rsd_token_logprobs");
}

int rsd_emitted_logprobs(const rsd_rows* target, int B, int num_nodes, int V, int L, const int32_t* accepted_len,
                         const int32_t* accepted_node, const int32_t* accepted_token, const int32_t* last_token, int K,
                         int32_t* out_token, float* out_logprob, float* out_entropy, int32_t* out_top_token,
                         float* out_top_logprob, int32_t* status, rsd_stream_t stream) {
    g_err[0] = 0;
    if (int e = check_vocab(V)) return e;
    if (L < 0 || num_nodes < 1 || num_nodes > RSD_MAX_TREE_NODES || L >= RSD_MAX_TREE_NODES) return fail(RSD_ERR_UNSUPPORTED, "L = %d, num_nodes = %d", L, num_nodes);
    if (int e = check_rows("target", target, V, num_nodes > 1)) return e;
    if (int e = check_entries("target", target)) return e;
    if (int e = check_batch(B, L + 1)) return e;
    if (K < 0 || K > RSD_MAX_K) return fail(RSD_ERR_UNSUPPORTED, "K = %d outside [0, %d]", K, (int)RSD_MAX_K);
    if (!accepted_len || !last_token || (L > 0 && (!accepted_node || !accepted_token)) || !out_logprob || !status || (K > 0 && (!out_top_token || !out_top_logprob)))
        return fail(RSD_ERR_INVALID_ARG, "null argument");
    if (B == 0) return RSD_OK;
    rsd::ScoreArgs a = score_args(target, L + 1, V, 1, K);
    a.num_rows = num_nodes;
    a.accepted_len = accepted_len; a.accepted_node = accepted_node; a.accepted_token = accepted_token; a.last_token = last_token;
    a.out_token = out_token; a.out_logprob = out_logprob; a.out_entropy = out_entropy; a.out_top_token = out_top_token; a.out_top_logprob = out_top_logprob;
    a.status = status;
    return launch_scores(target, B, a, (cudaStream_t)stream, "rsd_emitted_logprobs");
}

int rsd_token_logprobs_backward(const rsd_rows* rows, int B, int R, int V, const int32_t* token, int T, const float* grad_logprob,
                                const float* grad_entropy, void* grad_rows, int32_t* status, rsd_stream_t stream) {
    g_err[0] = 0;
    if (int e = check_vocab(V)) return e;
    if (int e = check_rows("rows", rows, V, R > 1)) return e;
    if (int e = check_entries("rows", rows)) return e;
    if (int e = check_batch(B, R)) return e;
    if (T < 1 || T > RSD_MAX_K) return fail(RSD_ERR_UNSUPPORTED, "T = %d outside [1, %d]", T, (int)RSD_MAX_K);
    if (!token || !grad_logprob || !grad_rows || !status) return fail(RSD_ERR_INVALID_ARG, "null argument");
    if (over_rows(rows, B, R, V, grad_rows, (int64_t)B * R * V * (rows->dtype == RSD_F32 ? 4 : 2))) return fail(RSD_ERR_INVALID_ARG, "grad_rows may not overlap the rows");
    if (B == 0) return RSD_OK;
    cudaStream_t s = (cudaStream_t)stream;
    rsd::ScoreArgs a = score_args(rows, R, V, T, 0);
    a.num_rows = R; a.token = token; a.g_logprob = grad_logprob; a.g_entropy = grad_entropy; a.grad = grad_rows; a.status = status;
    const bool aligned = rows_aligned(rows) && dense_aligned(grad_rows, V, rows->dtype);
    const unsigned slots = (unsigned)((int64_t)B * R);
    if (rows->dtype == RSD_F32) rsd::launch_score_grad_f32(aligned, slots, a, s);
    else rsd::launch_score_grad_bf16(aligned, slots, a, s);
    return check_launch("rsd_token_logprobs_backward");
}

int rsd_row_divergence(const rsd_rows* draft, const rsd_rows* target, int B, int R, int V, float* out_kl, float* out_reverse_kl,
                       float* out_overlap, int32_t* status, rsd_stream_t stream) {
    g_err[0] = 0;
    if (int e = check_pair(draft, target, B, R, V)) return e;
    if (!status || (!out_kl && !out_reverse_kl && !out_overlap)) return fail(RSD_ERR_INVALID_ARG, "null output");
    if (B == 0) return RSD_OK;
    cudaStream_t s = (cudaStream_t)stream;
    rsd::DivergenceArgs a = divergence_args(draft, target, R, V);
    a.out_kl = out_kl; a.out_reverse = out_reverse_kl; a.out_overlap = out_overlap; a.status = status;
    const bool aligned = rows_aligned(draft) && rows_aligned(target);
    const unsigned slots = (unsigned)((int64_t)B * R);
    if (draft->dtype == RSD_F32) rsd::launch_divergence_f32(aligned, slots, a, s);
    else rsd::launch_divergence_bf16(aligned, slots, a, s);
    return check_launch("rsd_row_divergence");
}

int rsd_row_divergence_backward(const rsd_rows* draft, const rsd_rows* target, int B, int R, int V, const float* grad_kl,
                                const float* grad_reverse_kl, void* grad_draft, int32_t* status, rsd_stream_t stream) {
    g_err[0] = 0;
    if (int e = check_pair(draft, target, B, R, V)) return e;
    if (!status || !grad_draft || (!grad_kl && !grad_reverse_kl)) return fail(RSD_ERR_INVALID_ARG, "null argument");
    const int64_t bytes = (int64_t)B * R * V * (draft->dtype == RSD_F32 ? 4 : 2);
    if (over_rows(draft, B, R, V, grad_draft, bytes) || over_rows(target, B, R, V, grad_draft, bytes)) return fail(RSD_ERR_INVALID_ARG, "grad_draft may not overlap the rows");
    if (B == 0) return RSD_OK;
    cudaStream_t s = (cudaStream_t)stream;
    rsd::DivergenceArgs a = divergence_args(draft, target, R, V);
    a.g_kl = grad_kl; a.g_reverse = grad_reverse_kl; a.grad = grad_draft; a.status = status;
    const bool aligned = rows_aligned(draft) && rows_aligned(target) && dense_aligned(grad_draft, V, draft->dtype);
    const unsigned slots = (unsigned)((int64_t)B * R);
    if (draft->dtype == RSD_F32) rsd::launch_divergence_grad_f32(aligned, slots, a, s);
    else rsd::launch_divergence_grad_bf16(aligned, slots, a, s);
    return check_launch("rsd_row_divergence_backward");
}

}  // extern "C"
