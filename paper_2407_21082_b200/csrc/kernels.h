// Internal launch interface between the C-ABI layer (api.cu) and the kernels.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

#include "eexit.h"

namespace ee {

constexpr int kMaxDevices = 64;

struct HeadArgs {
    const void* h;
    long long ld_h;
    const float* gamma;
    const float* beta;
    float ln_eps;
    const void* W;
    int M, d, V;
    const float* tau_per_row;
    float tau;
    int* argmax;
    float* entropy;
    float* maxprob;
    unsigned char* exit_mask;
    void* workspace;
    size_t workspace_bytes;
    cudaStream_t stream;
    int device;       // current device ordinal
    int num_sms;      // its multiprocessor count
    // Optional (tensor-core path, one head per launch): evaluate the rows h[row_idx[j]], j < *m_dev, instead of
    // rows 0 .. M-1; output row j belongs to input row row_idx[j], output rows at and beyond *m_dev are
    // meaningless.  Either may be NULL (identity / M).  Both are device pointers read after the stream's
    // earlier kernels have finished.
    const int* row_idx;
    const int* m_dev;
    // Optional (tensor-core path): fp32 [M], the difference between the two largest probabilities of each row.
    float* top2gap;
};

// ---- streaming kernel (fused LayerNorm + split-V mma.sync GEMV + last-CTA merge; up to four heads per launch) ----
constexpr int kStreamMaxCtas = 256;        // upper bound on the grid, used for workspace sizing
constexpr int kStreamMaxRows = 32;         // rows per launch (slab)
constexpr int kStreamMaxHeads = 4;
int stream_slab_rows(int d, int n_heads);  // rows one launch can take for this d (0 if d does not fit)
size_t stream_workspace_bytes(int n_heads);
ee_status stream_launch(const HeadArgs* heads, int n_heads);

// ---- skinny tensor-core kernel (one launch for up to four heads, weights as the MMA's M operand,
//      1 <= M <= 64, d % 64 == 0) ----
constexpr int kSkinnyMaxRows = 64;
constexpr int kSkinnyMaxHeads = 4;
bool skinny_supports(int M, int d);
size_t skinny_workspace_bytes(int n_heads);
// heads[0 .. n_heads) share M, d, V, ln_eps, workspace, stream and device; each has its own h, LayerNorm
// parameters, W, thresholds and outputs.
ee_status skinny_launch(const HeadArgs* heads, int n_heads);

// ---- tensor-core path (LayerNorm kernel, TMA + tcgen05 GEMM with fused statistics, merge): three launches
//      for up to four heads that share M, d, V, ln_eps, workspace, stream and device ----
constexpr int kGemmLaunchMaxHeads = 4;
int gemm_tile_n(int M, int V, int n_heads, int num_sms);   // vocabulary tile width used for M rows on num_sms SMs
size_t gemm_workspace_bytes(int M, int d, int V, int n_heads);
ee_status gemm_launch(const HeadArgs* heads, int n_heads);
// The same in two steps, for calls that are repeated: gemm_plan works out everything but the launches (tensor maps,
// tile width, launch shapes, instantiations) into `storage` (kGemmPlanBytes bytes, 8-byte aligned, plain data),
// gemm_run launches from it on `stream`.
constexpr size_t kGemmPlanBytes = 2048;
ee_status gemm_plan(const HeadArgs* heads, int n_heads, void* storage);
ee_status gemm_run(const void* storage, cudaStream_t stream);
int gemm_launches(int M, int n_heads);     // kernels one gemm_launch call starts

// ---- compaction and DSSD accept ----
ee_status compact_launch(const unsigned char* exit_mask, const void* h, long long ld_h, int M, int d,
                         int* kept_idx, int* kept_count, void* h_out, cudaStream_t stream);
ee_status accept_launch(const int* draft_tok, const unsigned char* draft_exit_mask, const int* verify_tok,
                        int S, int k, int kv, int* draft_len, int* accept_len, int* next_tok,
                        cudaStream_t stream);

ee_status compact_accept_launch(const unsigned char* exit_mask, const void* h, long long ld_h, int M, int d,
                                int* kept_idx, int* kept_count, void* h_out, const int* draft_tok,
                                const unsigned char* draft_exit_mask, const int* verify_tok, int S, int k, int kv,
                                int* draft_len, int* accept_len, int* next_tok, cudaStream_t stream);

// ---- calibration of a head's threshold (radix sort of the calibration tokens by entropy, scan, selection) ----
size_t calibrate_workspace_bytes(int n);
int calibrate_launches(int n);
ee_status calibrate_launch(const float* entropy, const int* argmax_head, const int* argmax_final, int n, double epsilon,
                           float* tau, int* counts, void* workspace, cudaStream_t stream);

// ---- KL divergence of a head's distribution from the teacher's, per token and mean (both logit sets fused) ----
size_t kl_workspace_bytes(int M, int d, int V);
ee_status kl_launch(const HeadArgs& head, const HeadArgs& teacher, const int* labels, float* kl, float* ce, float* loss);

// ---- cross-entropy of a head over the whole vocabulary, and its gradient ----
struct CeArgs {
    const void* h;
    long long ld_h;
    const float* gamma;
    const float* beta;
    float ln_eps;
    const void* W;
    int M, d, V;
    const int* labels;
    float* ce;             // forward outputs
    float* lse_out;
    float* loss_out;
    const float* lse;      // backward: what the forward call wrote, ce_in its ce or NULL
    const float* ce_in;
    const float* loss;
    const float* dce;
    const float* dloss;
    void* dh;
    long long ld_dh;
    void* dW;
    void* dgamma;
    void* dbeta;
    int accumulate;
    void* workspace;
    cudaStream_t stream;
    int device, num_sms;
};
size_t ce_workspace_bytes(int M, int d, int V, bool grad);
ee_status ce_launch(const CeArgs& a);
ee_status ce_grad_launch(const CeArgs& a);

// y bf16 [M][ld_y] in the column order of the 4-bit heads, ld_y = d rounded up to 64
ee_status layer_norm_permuted_launch(const void* h, long long ld_h, const float* gamma, const float* beta, float ln_eps, void* y, int ld_y,
                                     int M, int d, cudaStream_t stream);

// ---- heads with weights in 4 bits ----
size_t q4_weight_bytes(int V, int d, int group);
ee_status q4_pack_launch(const void* W, int V, int d, int group, void* q4, cudaStream_t stream);
ee_status q4_unpack_launch(const void* q4, int V, int d, int group, void* W, cudaStream_t stream);
size_t q4_head_workspace_bytes(int M, int d);
ee_status q4_head_launch(const HeadArgs& a, const void* q4, int group);      // a.W is not read

// ---- losses over the tokens of sequences ----
struct PolicyArgs {
    const float* ce;
    const float* old_ce;
    const float* ref_ce;       // NULL: no penalty
    const float* adv;          // per token, or per sequence where seq_start is given
    const int* labels;
    const int* seq_start;      // [S + 1] or NULL
    const float* counted;      // ee_head_ce's loss: [1] is the number of counted rows (read where seq_start is NULL)
    int M, V, S;
    double log_low, log_high;  // ln of the clip's borders
    float low, high;           // the borders
    float kl_weight;
    float* dce;
    float* loss;
    void* workspace;
};
struct PreferenceArgs {
    const float* ce;
    const float* ref_ce;       // NULL: none
    const int* labels;
    const int* seq_start;      // [2 P + 1]
    int M, V, P;
    float beta, smoothing;
    double share;              // of a pair: 1 / P
    float* dce;
    float* margin;
    float* loss;
    void* workspace;
};
size_t token_loss_workspace_bytes();
ee_status policy_loss_launch(const PolicyArgs& p, int num_sms, int device, cudaStream_t stream);
ee_status preference_loss_launch(const PreferenceArgs& p, int num_sms, int device, cudaStream_t stream);

// ---- norm over many tensors, and their scaling ----
size_t grad_norm_workspace_bytes(int n_tensors);
ee_status grad_norm_launch(const ee_tensor* tensors, int n_tensors, float* norm, void* workspace, int num_sms, cudaStream_t stream);
ee_status grad_clip_launch(const ee_tensor* tensors, void* const* out, int n_tensors, float max_norm, const float* norm, int num_sms,
                           cudaStream_t stream);

// ---- heads in microscaled 4-bit floating point ----
size_t fp4_weight_bytes(int V, int d, int group);
ee_status fp4_pack_launch(const void* W, int V, int d, int group, void* fp4, int num_sms, cudaStream_t stream);
ee_status fp4_unpack_launch(const void* fp4, int V, int d, int group, void* W, int num_sms, cudaStream_t stream);
size_t fp4_head_workspace_bytes(int M, int d, int V, int group);
ee_status fp4_head_launch(const HeadArgs& a, const void* fp4, int group);     // a.W is not read

// ---- embedding lookup and its gradient ----
ee_status embed_launch(const void* table, int V, int d, const int* tokens, int n, float scale, void* out, long long ld_out, int num_sms,
                       cudaStream_t stream);
size_t embed_grad_workspace_bytes(int n, int d, int V);
ee_status embed_grad_launch(const void* dout, long long ld_dout, const int* tokens, int n, int V, int d, float scale, void* dtable, int wide,
                            int accumulate, void* workspace, int num_sms, cudaStream_t stream);

// ---- stable radix sort of 64-bit words by `passes` digits of eight bits from bit `first_shift` on (calibrate.cu); a holds
//      the words, *sorted is a or b ----
size_t sort_words_scratch_bytes(int n);
ee_status sort_words_launch(unsigned long long* a, unsigned long long* b, int n, int first_shift, int passes, void* scratch,
                            const unsigned long long** sorted, cudaStream_t stream);

// ---- commit step of a DSSD round (k <= 32) ----
ee_status dssd_commit_launch(const int* draft_tok, const unsigned char* draft_exit_mask, const int* verify_tok, int S, int k,
                             int kv, int eos, int* out_tok, int cap, int* seq_len, unsigned char* finished, int* draft_len,
                             int* accept_len, int* next_tok, long long* stats, cudaStream_t stream);

// ---- a whole DSSD round driven from the host (drafting steps, verification pass, commit) ----
size_t dssd_round_layout_bytes(int S, int k, int d, int n_draft_heads, size_t head_ws_bytes);
ee_status dssd_round_run(const ee_dssd_round_args& a, const ee_head* draft_heads, int n_draft_heads, size_t head_ws_bytes);

// ---- diagnostic: a bounded wait that is made to give up ----
int hidden_from_tables(const ee_hidden_tables* m, const int* tokens, int n_rows, int which, void* h_out, cudaStream_t stream);
ee_status selftest_wait_timeout_launch(void* workspace, cudaStream_t stream);
ee_status selftest_read_stream_launch(const void* src, size_t bytes, void* workspace, int num_sms, cudaStream_t stream);

// ---- one step of the cascade of heads: rows answered by head k are recorded, the others move on ----
int cascade_select_max_rows();
ee_status cascade_select_launch(const unsigned char* mask0, const int* argmax0, const float* entropy0, size_t stride, int M,
                                int k0, int n, int n_heads, int* exit_head, int* token, float* entropy_out, int* rows_in,
                                cudaStream_t stream);
ee_status cascade_step_launch(const unsigned char* exit_mask, const int* argmax, const float* entropy,
                              const int* idx_in, const int* m_in, int M, int k, int is_last, int n_heads,
                              int* exit_head, int* token, float* entropy_out, int* idx_out, int* m_out, int* rows_in,
                              cudaStream_t stream);

}  // namespace ee
