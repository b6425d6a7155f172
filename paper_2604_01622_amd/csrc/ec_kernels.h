// Internal launchers of the expert-choice MoE kernels.  Each returns the
// hipError_t of its launch(es); all work goes on the given stream.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "row_split.h"

namespace ec {

enum { DT_F32 = 0, DT_BF16 = 1 };

// Groups handled by one top-k launch (the table travels as a kernel argument).
constexpr int TOPK_MAX_GROUPS = 128;

struct GroupTable {
  int n;                            // groups in this launch
  int off[TOPK_MAX_GROUPS];         // first token of the group
  int len[TOPK_MAX_GROUPS];         // tokens in the group
  int k[TOPK_MAX_GROUPS];           // tokens each expert takes from the group
  int seg[TOPK_MAX_GROUPS];         // first row of the group's segment in an expert buffer
};

// S [N,E] and ST [E,N] fp32 from X [N,d] and Wg [E,d].  ST null (token choice): no transposed
// copy, and experts of equal logits get equal scores to the bit.
hipError_t launch_router_softmax(int dtype, const void* X, const void* Wg, float* S, float* ST,
                                 int N, int d, int E, float inv_tau, hipStream_t st);

// Column top-k of ST per (group, expert): sel_token/sel_gate [E,K], slotT [E,N].
hipError_t launch_topk(const float* ST, int N, int E, int K, const GroupTable& tab,
                       int32_t* sel_token, float* sel_gate, int32_t* slotT, hipStream_t st);

// Xe[r, :] = X[sel_token[r], :] for all rows.
hipError_t launch_gather(int dtype, const void* X, const int32_t* sel_token, void* Xe,
                         long rows, int d, int N, hipStream_t st);

// Y[i, :] = Xr[i, :] (if Xr) + sum_j S[i,j] O[j kstride + slotT[j,i], :] over experts j
// with 0 <= slotT[j,i] < K (Xr may alias Y); kstride < 0 means K (one buffer of K
// rows per expert), 0 means slot holds rows of one packed buffer.
hipError_t launch_combine(int dtype, const void* O, const float* S, const int32_t* slotT,
                          const void* Xr, void* Y, int N, int E, int K, int d, hipStream_t st,
                          long kstride = -1);

// Dropout of a call: an element whose 16-bit draw is below thr is dropped, the others are
// scaled (thr 0: none is drawn); rng: device [2], the seed and the offset (see dropout.h).
struct Dropout {
  uint32_t thr;
  float scale;
  const uint64_t* rng;
};

// The combine of token-choice training: Y = R + dropout(Xr + sum_j O[slotT[j, i]]) over the
// packed rows (R and Xr may be null; Xr may alias Y).
hipError_t launch_combine_drop(int dtype, const void* O, const int32_t* slotT, const void* Xr,
                               const void* R, const Dropout& drop, void* Y, int N, int E,
                               int max_rows, int d, hipStream_t st);

// Y = R + dropout(X) over n elements (R may be null; Y may be X or R).
hipError_t launch_dropout(int dtype, const void* X, const void* R, const Dropout& drop, void* Y,
                          long n, hipStream_t st);

// Backward combine: dX[i,:] = Xr[i,:] + sum_j dXe[j, slotT[j,i], :]  (Xr may alias dX).
// kstride as for launch_combine.
hipError_t launch_bwd_combine(int dtype, const void* dXe, const int32_t* slotT, const void* Xr,
                              void* dX, int N, int E, int K, int d, hipStream_t st,
                              long kstride = -1);

// Router backward, part 1: dZ = S * (dS - <S, dS>) / tau  [N, EP] in the storage type
// (columns E..EP-1 zero), from S_ij dS_ij = sum over q of dsp[(j K + slot_ij) nparts + q]
// on the selection (0 elsewhere).
hipError_t launch_router_dz(int dtype, const float* S, const float* dsp, int nparts,
                            const int32_t* slotT, void* dZ, int N, int E, int EP, int K,
                            float inv_tau, hipStream_t st);

// Router backward, part 2: dX = dZ Wg.
hipError_t launch_router_dx(int dtype, const void* dZ, const void* Wg, void* dX, int N, int E,
                            int EP, int d, hipStream_t st);

// Router backward, part 3: dWg [E,d] fp32 = dZ^T X, split over the tokens into at most
// `splits` (router_dwg_splits) partial sums (part [splits,E,d] fp32) added in a fixed order.
hipError_t launch_router_dwg(int dtype, const void* dZ, const void* X, float* dWg, float* part,
                             int splits, int N, int E, int EP, int d, hipStream_t st);

// ---- grouped GEMMs over E experts (M = K rows per expert) ----

// H = Xe W1^T, Xe W3^T -> A = SiLU(H1) * H3 (and H1, H3 if non-null).
// `shared`: the same product for the shared experts (own kernel symbol).
// rows (routed experts, may be null): Xe is then X itself and row m of
// expert e reads X[rows[e M + m]] (the gather happens in the operand load).
// gate (may be null): [E, M] fp32, row m of expert e is written as
// A = gate[e M + m] SiLU(H1) H3 (H1, H3 themselves unscaled); scale: every row's factor
// without gate.
hipError_t launch_gemm_w13(int dtype, const void* Xe, const void* W1, const void* W3, void* A,
                           void* H1, void* H3, int E, int M, int d, int h, hipStream_t st,
                           bool shared = false, const int32_t* rows = nullptr,
                           const float* gate = nullptr, float scale = 1.f);
// O = A W2^T.
hipError_t launch_gemm_w2(int dtype, const void* A, const void* W2, void* O, int E, int M, int d,
                          int h, hipStream_t st, bool shared = false);
// dA = g dO W2 and the SwiGLU backward: dH[:, 0:h] = dH1, dH[:, h:2h] = dH3
// ([E,M,2h]), g = gate[e M + m] per row (scale when gate is null); W2 is read
// K-major.  dsp (may be null):
// [E M, dsp_parts(dtype, h)] fp32, per row and column block the sum of dA * A
// (A = SiLU(H1) H3), whose row sum is the gate's gradient times the gate when
// dO holds the rows of dY.  rows (may be null): dO is then dY itself and
// row m of expert e reads dY[rows[e M + m]].
hipError_t launch_gemm_dA(int dtype, const void* dO, const void* W2, const void* H1,
                          const void* H3, void* dH, int E, int M, int d, int h, hipStream_t st,
                          bool shared = false, float* dsp = nullptr, const int32_t* rows = nullptr,
                          const float* gate = nullptr, float scale = 1.f);
// gate-gradient partials per row of the dA product (blocks of 128 columns of
// d_ff in bf16, 64 in fp32)
int dsp_parts(int dtype, int h);
// dXe = dH1 W1 + dH3 W3  ([E,M,d]).
// shared: dXe += dH1 W1 + dH3 W3 (the shared experts' term added to dX).
// The weights are read K-major (bf16: h a multiple of 64).
hipError_t launch_gemm_dXe(int dtype, const void* dH, const void* W1, const void* W3, void* dXe,
                           int E, int M, int d, int h, hipStream_t st, bool shared = false);
// dW2 = dO^T A  ([E,d,h]).  rows (may be null): dO is then dY itself and
// row m of expert e reads dY[rows[e M + m]] (the gather happens in the loads).
hipError_t launch_gemm_dW2(int dtype, const void* dO, const void* A, void* dW2, int E, int M,
                           int d, int h, hipStream_t st, const int32_t* rows = nullptr);
// dW1 = dH1^T Xe, dW3 = dH3^T Xe  ([E,h,d] each).  rows (bf16, may be null): Xe
// is then X itself and row m of expert e reads X[rows[e M + m]].
hipError_t launch_gemm_dW13(int dtype, const void* dH, const void* Xe, void* dW1, void* dW3,
                            int E, int M, int d, int h, hipStream_t st,
                            const int32_t* rows = nullptr);

// Token drop statistic: cnt[i] = #{j : slotT[j, i] >= 0} for i < N, then
// dropped[g] = #{i in group g : cnt[i] == 0} for the tab.n groups of the table.
hipError_t launch_coverage_count(const int32_t* slotT, int N, int E, int32_t* cnt,
                                 hipStream_t st);
hipError_t launch_coverage_drop(const int32_t* cnt, const GroupTable& tab, int32_t* dropped,
                                hipStream_t st);

// Shared experts' weight gradients (one batch of N rows, K-major operands):
// dW2 = dY^T A ([d,h]) and [dW1; dW3] = dH^T X ([h,d] each), split over the
// rows into at most `splits` (wgrad_splits) fp32 partials (part: splits * max(d*h, 2*h*d) floats)
// added in a fixed order.
hipError_t launch_shared_dW2(int dtype, const void* dY, const void* A, void* dW2, int N, int d,
                             int h, float* part, int splits, hipStream_t st);
hipError_t launch_shared_dW13(int dtype, const void* dH, const void* X, void* dW1, void* dW3,
                              int N, int d, int h, float* part, int splits, hipStream_t st);

// ---- token choice (the comparison policy): packed, data-dependent expert loads ----

// G [N,E]: normalised gates of each token's top-k experts; flagT [E,N]: 1 if chosen.
hipError_t launch_tc_topk(const float* S, int N, int E, int k, float* G, int32_t* flagT,
                          hipStream_t st);
// cnt[(g0+g) E + j] = min(tokens of group g that chose j, cap_g) for the table's groups.
hipError_t launch_tc_count(const int32_t* flagT, int N, int E, const GroupTable& tab, int g0,
                           int32_t* cnt, hipStream_t st);
// Packed row offsets rows [E+1] and per-(group, expert) row offsets seg [G,E]; order [E, 4]
// (training; may be null): the experts as the products that contract over an expert's rows
// take them, each with its first row and its number of rows.
hipError_t launch_tc_offsets(const int32_t* cnt, int G, int E, int32_t* rows, int32_t* seg,
                             int32_t* order, hipStream_t st);
// slotT: choice flags in, packed rows (-1: not kept) out; sel[row] = token.  Without
// sel_gate G is zeroed on dropped pairs; with it (training) sel_gate[row] = scale G of the
// pair and G keeps the gates of every choice.
hipError_t launch_tc_place(int32_t* slotT, float* G, int N, int E, const GroupTable& tab, int g0,
                           const int32_t* seg, int32_t* sel, float* sel_gate, float scale,
                           hipStream_t st);
// The forward products over packed rows: expert e owns rows [rows[e], rows[e+1]), max_rows
// of all experts and max_rows_per_expert of each at most.
// sel (may be null): Xe is then X itself and packed row r reads X[sel[r]].
// gate (may be null): [max_rows] fp32, packed row r is written as A = gate[r] SiLU(H1) H3.
// H1, H3 (may be null): [max_rows, h], the projections themselves.
hipError_t launch_gemm_w13_var(int dtype, const void* Xe, const void* W1, const void* W3, void* A,
                               void* H1, void* H3, int E, const int32_t* rows, long max_rows,
                               int max_rows_per_expert, int d, int h, hipStream_t st,
                               const int32_t* sel = nullptr, const float* gate = nullptr);
hipError_t launch_gemm_w2_var(int dtype, const void* A, const void* W2, void* O, int E,
                              const int32_t* rows, long max_rows,
                              int max_rows_per_expert, int d, int h, hipStream_t st);
// The backward products over packed rows (conventions of launch_gemm_dA, _dXe, _dW2 and
// _dW13): sel[r] is the token of packed row r, whose rows of dY (dA, dW2) and X (dW13) the
// products read themselves.  dH [max_rows, 2h], dsp [max_rows, dsp_parts(dtype, h)].  An
// expert without rows gets zero weight gradients.  order [E, 4]: the experts as the
// weight gradients take them (launch_tc_offsets).
hipError_t launch_gemm_dA_var(int dtype, const void* dY, const void* W2, const void* H1,
                              const void* H3, void* dH, float* dsp, int E, const int32_t* rows,
                              long max_rows, int max_rows_per_expert, int d, int h,
                              const int32_t* sel, const float* gate, hipStream_t st);
hipError_t launch_gemm_dXe_var(int dtype, const void* dH, const void* W1, const void* W3,
                               void* dXe, int E, const int32_t* rows, long max_rows,
                               int max_rows_per_expert, int d, int h, hipStream_t st);
hipError_t launch_gemm_dW2_var(int dtype, const void* dY, const void* A, void* dW2, int E,
                               const int32_t* order, long max_rows,
                               int max_rows_per_expert, int d, int h, const int32_t* sel,
                               hipStream_t st);
hipError_t launch_gemm_dW13_var(int dtype, const void* dH, const void* X, void* dW1, void* dW3,
                                int E, const int32_t* order, long max_rows,
                                int max_rows_per_expert, int d, int h, const int32_t* sel,
                                hipStream_t st);

// ---- the balance loss of token choice ----

// The tokens of the table's groups go in chunks of `chunk`; tab.seg[g] is the first chunk
// of group g in the launch and tab.seg[n] their number.
struct ChunkTable {
  int n;
  int chunk;
  int off[TOPK_MAX_GROUPS];
  int len[TOPK_MAX_GROUPS];
  int cap[TOPK_MAX_GROUPS];
  int seg[TOPK_MAX_GROUPS + 1];
};
// Tokens of a chunk, for N tokens; where no group has more than BALANCE_WHOLE, each is one
// chunk and launch_balance_partial finishes it.
constexpr int BALANCE_WHOLE = 256;
int balance_chunk(int N);
// ... of launch_balance_backward and launch_tc_router_dz, and of launch_tc_choose.
int balance_backward_chunk(int N);
constexpr int TC_CHOOSE_CHUNK = 64;
// What the sums' kernel leaves for launch_balance_finish (chunks and groups of one launch).
struct BalanceSums {
  double* psum;      // [chunks, E]
  int32_t* pcnt;     // [chunks, E]
  double* part;      // [groups, ceil(E / 64)] parts of the loss
  int32_t* done;     // [groups]
};
// Sums of S and the number of choices among each row's k largest (ties: the lower index),
// per chunk: psum, pcnt [seg[n], E]; whole: loss [n] and counts [n, E] instead.
hipError_t launch_balance_partial(const float* S, int E, int k, const ChunkTable& tab, bool whole,
                                  const BalanceSums& sums, float* loss, int32_t* counts,
                                  hipStream_t st);
// The same sums in one pass with launch_tc_topk's outputs.
hipError_t launch_tc_choose(const float* S, int N, int E, int k, const ChunkTable& tab,
                            const BalanceSums& sums, float* G, int32_t* flagT, hipStream_t st);
// counts [n, E] and loss [n] of the table's groups from their chunks' sums (counts2: a
// second copy of the counts, kept: the counts capped at tab.cap, unless null).
hipError_t launch_balance_finish(const BalanceSums& sums, int E, int k, const ChunkTable& tab,
                                 float* loss, int32_t* counts, int32_t* counts2, int32_t* kept,
                                 hipStream_t st);
// dZ [N, E] fp32 of the table's groups: the loss's gradient in the logits (counts [n, E] and
// dloss [n] of these groups).
hipError_t launch_balance_backward(const float* S, const int32_t* counts, const float* dloss,
                                   int E, int k, float inv_tau, const ChunkTable& tab, float* dZ,
                                   hipStream_t st);
// The router's dZ [N, EP] (storage type, columns E.. zero) of token-choice training for the
// table's groups: the gates' gradient, u - G sum_j u with u_ij the sum of the partials of
// packed row slotT[j, i] < max_rows (0 where it is -1), plus the balance loss's with
// dloss (null: none).
hipError_t launch_tc_router_dz(int dtype, const float* S, const float* G, const int32_t* slotT,
                               const float* dsp, int nparts, const int32_t* counts,
                               const float* dloss, void* dZ, int N, int E, int EP, int k,
                               int max_rows, float inv_tau, const ChunkTable& tab,
                               hipStream_t st);

// Fill n int32/fp32/bytes with zero (a kernel, not a memset node).
hipError_t launch_zero(void* p, size_t bytes, hipStream_t st);


}  // namespace ec
