// Internal launcher declarations between the C ABI layer and the kernel files.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace lmbp {

enum { kGelu = 0, kSilu = 1 };

constexpr int kXcds = 8;          // consecutive blocks go to them in turn
constexpr int kMaxDevices = 64;   // of one process

// HIP takes fewer than 2^32 threads to a grid dimension. A launch of more reports success and runs
// their number modulo 2^32 (measured), so where the number of blocks grows with the data the launch goes
// out in parts: f(first, count) launches units first .. first + count - 1, at most `part` of them.
constexpr int64_t most_blocks(int threads) { return int64_t(0xffffffff) / threads; }
template <class F>
hipError_t in_parts(int64_t count, int64_t part, F f) {
  for (int64_t first = 0; first < count; first += part) {
    f(first, std::min(part, count - first));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The current device and its CU count (queried once per device).
hipError_t current_device(int& dev, int& cus);

// Runtime tables of a general family member (kernel argument, passed by value):
// thresholds t[0..2^k-2] as fp32 round-down values, levels lv[0..2^k-1] in fp32.
struct StepTable {
  float t[15];
  float lv[16];
};

hipError_t launch_act_fwd(int act, bool bf16, int64_t n, const void* x, void* y,
                          uint32_t* codes, bool vec_ok, hipStream_t s);
hipError_t launch_act_bwd(int act, bool bf16, int64_t n, const void* dy, const uint32_t* codes,
                          void* dx, bool vec_ok, hipStream_t s);

// Gated form h = act(g) * u (only act = kSilu is instantiated).
hipError_t launch_glu_fwd(int act, bool bf16, int64_t n, const void* g, const void* u, void* h,
                          void* s, uint32_t* codes, bool vec_ok, hipStream_t st);
hipError_t launch_glu_bwd(int act, bool bf16, int64_t n, const void* dh, const void* u,
                          const void* s, const uint32_t* codes, void* dg, void* du, bool vec_ok,
                          hipStream_t st);

// vec_ok: every tensor pointer 16-byte aligned and cols * element bytes a
// multiple of 16 (each row starts on a vector boundary).
hipError_t launch_norm_fwd(bool ln, bool bf16, int64_t rows, int64_t cols, float eps,
                           const void* x, void* z, float* rstd, bool vec_ok, hipStream_t s);
hipError_t launch_norm_bwd(bool ln, bool bf16, int64_t rows, int64_t cols, const void* dz,
                           const void* z, const float* rstd, void* dx, bool vec_ok,
                           hipStream_t s);

hipError_t launch_stepact_fwd(int act, int bits, bool bf16, int64_t n, const void* x, void* y,
                              uint32_t* codes, bool vec_ok, const StepTable& tab, hipStream_t s);
hipError_t launch_stepact_bwd(int bits, bool bf16, int64_t n, const void* dy, const uint32_t* codes,
                              void* dx, bool vec_ok, const StepTable& tab, hipStream_t s);

// z = bf16(x W^T + bias) (bf16 operands, fp32 accumulation); y = act(z), codes of z;
// z stored when non-null. N % 16 == 0, K % 8 == 0, x/w/y/z 16-byte aligned.
hipError_t launch_linear_act_fwd(int act, int64_t M, int64_t N, int64_t K, const void* x,
                                 const void* w, const void* bias, void* y, uint32_t* codes,
                                 void* z, hipStream_t s);

// Gated form: g = bf16(x Wg^T), u = bf16(x Wu^T); h = SiLU(g) * u, s = SiLU(g), u stored,
// codes of g; g stored when non-null. Same requirements as launch_linear_act_fwd.
hipError_t launch_linear_glu_fwd(int64_t M, int64_t N, int64_t K, const void* x, const void* w_gate,
                                 const void* w_up, void* h, void* s_out, void* u, uint32_t* codes,
                                 void* g, hipStream_t s);

// The same layers with MS-RMSNorm in front (Sec. 5.2 eq. norm_linear): x [M x K] is the
// norm's input. The norm kernel writes rstd (fp32, per row) and the norm's output z_norm
// [M x K]; the GEMM runs on x and scales each row's fp32 sums by its rstd before the
// bias. pre / g: the rounded pre-activation (gate), stored when non-null. x, w, z_norm
// 16-byte aligned; K % 8 == 0, N % 16 == 0.
hipError_t launch_linear_rms_act_fwd(int act, int64_t M, int64_t N, int64_t K, float eps,
                                     const void* x, const void* w, const void* bias, void* y,
                                     uint32_t* codes, void* pre, void* z_norm, float* rstd,
                                     hipStream_t s);
hipError_t launch_linear_rms_glu_fwd(int64_t M, int64_t N, int64_t K, float eps, const void* x,
                                     const void* w_gate, const void* w_up, void* h, void* s_out,
                                     void* u, uint32_t* codes, void* g, void* z_norm, float* rstd,
                                     hipStream_t s);

// The form that the fused forward of a layer runs in on the current device (256 CUs without
// one): 0, 1 split-K with 16, 32 rows; 2 .. 5 tiles of 256 x 256, 128 x 256, 128 x 128, 64 x
// 128; and the most tiles that a block computes.
struct LinearForm {
  int form;
  int64_t rounds;
};
LinearForm linear_form(bool gated, int64_t M, int64_t N, int64_t K);

// How dW is computed on the current device (256 CUs without one): made once per call, for K =
// 0 if dw is not asked for.
struct LinearGradPlan {
  int tile = 0;        // 0: 256 x 256, 1: 128 x 256, 2: 128 x 128
  int64_t splits = 1;  // shares of the rows that hold any
  int64_t per = 1;     // 64-row steps per share
};
LinearGradPlan linear_grad_plan(int64_t M, int64_t N, int64_t K);
size_t linear_grad_workspace(int64_t M, int64_t N, int64_t K, bool bias, const LinearGradPlan& plan);
// The tile of dW (0 .. 2: 256 x 256, 128 x 256, 128 x 128), the shares that its rows are split
// into, and the most units of work that a block takes.
struct LinearGradForm {
  int tile;
  int64_t splits, rounds;
};
LinearGradForm linear_grad_form(int64_t M, int64_t N, int64_t K);

// Backward of a fused linear layer's parameters. db non-null: dz = dy slope[code] is
// computed here (act) and db is the column sums of dz; else dz is an input. dw non-null:
// dw = bf16(dz^T x). Workspace of linear_grad_workspace bytes (same sizes and plan; bias: db
// non-null; K = 0 if dw is null). N % 16 == 0, K % 8 == 0, every tensor 16-byte aligned, db 2-byte
// aligned.
hipError_t launch_linear_grad(int act, int64_t M, int64_t N, int64_t K, const void* dy, const uint32_t* codes,
                              const void* x, void* dz, void* dw, void* db, void* workspace,
                              const LinearGradPlan& plan, hipStream_t s);

// Rows in 8 bits (q8_device.hpp). columns: null, or a factor per column that x is multiplied by
// first; pitch >= cols: bytes from one row of q to the next, zeros written behind each row.
hipError_t launch_q8_rows(bool bf16, int64_t rows, int64_t cols, int64_t pitch, const void* x, const float* columns,
                          int8_t* q, float* scale, hipStream_t s);
hipError_t launch_q8_values(bool bf16, int64_t rows, int64_t cols, const int8_t* q, const float* scale, void* v,
                            hipStream_t s);
// MS-RMSNorm of x, or of sum = x + res (res and sum both null or both given), in 8 bits.
hipError_t launch_msrms_q8_fwd(bool bf16, int64_t rows, int64_t cols, float eps, const void* x, const void* res,
                               void* sum, int8_t* q, float* scale, float* rstd, hipStream_t s);
// dz_bf16: the type of dz; bf16 that of ds and dx (not fp32 with a bf16 dz).
hipError_t launch_msrms_q8_bwd(bool dz_bf16, bool bf16, int64_t rows, int64_t cols, const void* dz, const int8_t* q,
                               const float* scale, const float* rstd, const void* ds, void* dx, hipStream_t s);

// Linear layers of 8-bit rows and weights; bf16: the type of y and bias, or of dy; dx_bf16 that of
// add (may be null, or dx) and dx. No more than kQ8MaxDepth products to a sum: 128 * 128 * kQ8MaxDepth < 2^31. Workspaces of
// the functions' bytes, 16-byte aligned.
constexpr int64_t kQ8MaxDepth = 131071;
hipError_t launch_linear_q8_fwd(bool bf16, int64_t M, int64_t N, int64_t K, const int8_t* q, const float* scale,
                                const int8_t* w, const float* w_scale, const void* bias, void* y, void* workspace,
                                hipStream_t s);
size_t linear_q8_fwd_workspace(int64_t M, int64_t N, int64_t K);
size_t linear_q8_bwd_workspace(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear_q8_bwd(bool bf16, bool dx_bf16, int64_t M, int64_t N, int64_t K, const void* dy, const int8_t* w,
                                const float* w_scale, const void* add, void* dx, void* workspace, hipStream_t s);

// The form that aligned tensors of these sizes take on the current device (256 CUs without one): 0
// dot products, 1 .. 3 split-K with 16, 32, 64 rows to a block, 4 .. 7 tiles of 64 x 128, 128 x
// 128, 128 x 256, 256 x 256, 8 the general form; the blocks that share a sum's length; whether rows
// are copied to aligned ones first.
struct LinearQ8Form {
  int form, shares;
  bool copies;
};
LinearQ8Form linear_q8_fwd_form(int64_t M, int64_t N, int64_t K);
LinearQ8Form linear_q8_bwd_form(int64_t M, int64_t N, int64_t K);

// Sums over the rows of dy; db_bf16: the type of db. A workspace of the function's bytes, 16-byte aligned.
size_t linear_bias_grad_workspace(int64_t m, int64_t n);
hipError_t launch_linear_bias_grad(bool bf16, bool db_bf16, int64_t m, int64_t n, const void* dy, void* db, void* workspace,
                                   hipStream_t s);

// A tensor of heads: elements from row to row and from head to head; a head's columns lie together.
struct HeadsView {
  void* p = nullptr;
  int64_t row = 0, head = 0;
};

// Rotary positions (rope_kernels.hip): up to kRopePairs pairs of kRopeDim columns, freqs and axes in host memory.
constexpr int kRopePairs = 256, kRopeDim = 512;
struct RopePlan {
  int64_t tokens, dim, pairs;
  int64_t heads[2];        // of queries and keys, not both 0
  const void* positions;   // [axes][tokens], 4 or (wide) 8 bytes each
  int64_t axis_stride;
  const double* freqs;     // [pairs], finite
  const int32_t* axes;     // [pairs] or null
  bool wide, interleaved;
};
hipError_t launch_rope(bool bf16, const RopePlan& r, bool back, const HeadsView (&x)[2], const HeadsView (&y)[2], hipStream_t s);
hipError_t launch_msrms_rope_fwd(bool bf16, const RopePlan& r, float eps, bool gain_bf16, const void* const (&gain)[2],
                                 const HeadsView (&x)[2], const HeadsView (&y)[2], float* const (&rstd)[2], hipStream_t s);
// kept: y without gains, x with. dgain and the workspace (msrms_rope_bwd_workspace bytes) only with gains.
size_t msrms_rope_bwd_workspace(int64_t dim);
hipError_t launch_msrms_rope_bwd(bool bf16, const RopePlan& r, bool gain_bf16, const void* const (&gain)[2], const HeadsView (&dy)[2],
                                 const HeadsView (&kept)[2], const float* const (&rstd)[2], const HeadsView (&dx)[2],
                                 void* const (&dgain)[2], void* workspace, hipStream_t s);

// Attention (bf16). rows of all sequences one behind the other; starts null: batch sequences of one length.
struct AttentionPlan {
  int64_t batch, heads, kv_heads, dim, q_rows, k_rows;
  const int32_t *q_starts, *k_starts, *k_lens;
  bool causal, fill;
  float scale;
};
constexpr int kAttentionDim = 128;   // widest head
size_t attention_fwd_workspace(const AttentionPlan& a);
hipError_t launch_attention_fwd(const AttentionPlan& a, const HeadsView& q, const HeadsView& k, const HeadsView& v, const HeadsView& o,
                                float* lse, void* workspace, hipStream_t s);
size_t attention_bwd_workspace(const AttentionPlan& a);
hipError_t launch_attention_bwd(const AttentionPlan& a, const HeadsView& d_o, const HeadsView& q, const HeadsView& k, const HeadsView& v,
                                const HeadsView& o, const float* lse, const HeadsView& dq, const HeadsView& dk, const HeadsView& dv,
                                void* workspace, hipStream_t s);

hipError_t launch_copy(const void* src, void* dst, int64_t bytes, hipStream_t s);

}  // namespace lmbp
