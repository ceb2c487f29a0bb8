// The LM-head contractions of one slab of tokens, as the loss calls use them: logits with exp-logits
// and log-sum-exp, and the backward GEMMs (lmhead.hip).
#pragma once
#include "common.h"

namespace fastrl {

// What a call's slabs share.
struct LmCall {
  const void* hidden;
  const int32_t* row_index;
  const void* W;
  int32_t dtype, d, V;
  int64_t T;
  void* dhidden;            // [T][d] (NULL: not computed)
  int32_t dhidden_dtype;
  void* dW;                 // [V][d] (NULL: not computed)
  int32_t dW_dtype;         // FASTRL_BF16: written once, from bf16 operands only
  int64_t tcp;              // tokens that the per-token arrays hold: the largest slab's, a multiple of 256
  float zscale;             // logits are multiplied by it (0: not)
};

// Workspace of a slab.
struct LmWs {
  void *WT = nullptr, *E1 = nullptr, *Bd = nullptr;
  float *pmax = nullptr, *psum = nullptr, *psz = nullptr, *zlab = nullptr, *shift = nullptr, *cslab = nullptr;
  int32_t *yslab = nullptr, *redo_blk = nullptr, *redo_count = nullptr;
  // NULL, or sum exp(z - s_t) of each token; without a gradient asked for, s_t (shift) is the token's maximum then
  float* sum = nullptr;
  // NULL, or given ids, a row of pick_n per slab token: ascending, where those of each 256 vocabulary rows begin
  // (and, last, end) and their logits
  const int32_t* pick_ids = nullptr;
  const uint8_t* pick_off = nullptr;
  float* pick_z = nullptr;
  int32_t pick_n = 0, pick_ldo = 0;
};

// Bytes of the region WT of a call whose slabs hold the given tokens: W^T, or the float32 parts that
// dhidden is summed from.
int64_t lm_wt_bytes(const LmCall& a, const int64_t* slab_tokens, size_t nslab);

// W^T, once a call, where dhidden is computed from it.
int lm_prepare(const LmCall& a, const LmWs& w, hipStream_t stream);

// Logits of tokens t0 .. t0 + Tc: lse, logp (and entropy, with w.psz) into the given arrays of all
// tokens; with a gradient asked for also the exp-logits E1 and the shifts.  Needs w.yslab and cleared
// w.shift and flags; rows that w.shift marks have new partials that are not merged yet.
int lm_forward(const LmCall& a, const LmWs& w, int64_t t0, int32_t Tc, float* lse, float* logp,
               float* ent, hipStream_t stream);

// dhidden rows and dW from E1 and c_t (w.cslab): dH = -c E W, dW (+)= -(c E)^T H.
int lm_backward(const LmCall& a, const LmWs& w, int64_t t0, int32_t Tc, bool dW_add,
                hipStream_t stream);

// redo_any flag of a slab (nonzero iff a row was marked)
inline int32_t* lm_redo_any(const LmWs& w, int32_t Tc) { return w.redo_blk + (Tc + 255) / 256; }

}  // namespace fastrl
