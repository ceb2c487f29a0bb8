// Distillation from a teacher's top logits, forward and backward, fused with the student's LM head.
//
// For kept token t with the teacher's entries (y_k, a_k) and temperature tau:
//   q_k = exp(a_k / tau - L),  L = log sum_k exp(a_k / tau) or the teacher's own log-sum-exp
//   l = log sum_v exp(z_v / tau),  z = h W^T,  log p_k = z_{y_k} / tau - l
//   token_t = sum_k q_k (log q_k - log p_k),   loss = c sum_t w_t token_t
//   dz_v = gamma (Q p_v - sum_{k: y_k = v} q_k),  gamma = c w_t / tau,  Q = sum_k q_k
// The slab engine of the policy loss (lmhead.h) stores E_v = exp(z_v / tau - s) and takes dH = -c E W,
// dW = -(c E)^T H.  With c = -gamma Q exp(s - l) the rows of E hold dz but for the teacher's entries,
//   E_{y_k} <- (p_k - q_k / Q) exp(l - s),
// formed here in 64 bits from the float32 logit, so that where the student has come close to the
// teacher the small difference is rounded once, and not two large terms.
//
// Roundings to bf16 (bf16 operands, whatever the gradients' type): E, and in dW c h, operands of 16-bit matrix
// products; then a bf16 result once, from float32 sums.  Against 64 bits, relative: dhidden 0.0024, dW 0.0029 (a
// float32 computation rounded once: 0.0017); in calls of one token, where a few entries of E can hold the whole
// gradient, up to 0.0035 and 0.0038.  c h would be exact for a power of two c, which needs l before E is
// written; E scaled by what is left of c afterwards would be rounded again, in a pass that costs 6%; float16 operands
// lack the range of exp(z / tau).
#include <algorithm>
#include <cmath>
#include <string>

#include "gemm_loop.h"
#include "lmhead.h"

namespace fastrl {

constexpr int kMaxDistill = 128;            // entries per token
constexpr int64_t kDistillSlab = 32768;     // tokens per slab
constexpr int32_t kAbsent = 0x7fffffff;     // id of an entry that does not count

struct DistillParams {
  int32_t V, K;
  int64_t t0;             // first token of the slab
  int32_t Tc;
  const int32_t* ids;     // [T][K]
  const float* a;         // [T][K]
  const float* tlse;      // [T] or NULL
  const float* weight;    // [T] or NULL
  double w_default, loss_scale;
  float zscale;           // 1 / tau
  int32_t* sid;           // [Tc][K] the entries by ascending id
  float* sa;
  uint8_t* off;           // [Tc][nmb + 1] first of them in each vocabulary block
  float* zk;              // [Tc][K] their logits over tau
  float* lse;             // [T]
  float* token_loss;      // [T]
  double* term;           // [T] of the loss
  float* cslab;           // [Tc]
  void* E;                // NULL without a backward
  int64_t ldE;
  int32_t bf16;
  const float* shift;     // of the slab (without a backward: the token's maximum of z / tau)
  const float* sum;       // [Tc] sum exp(z / tau - s)
  const float* pmax;      // [nmb][ldp] maxima of the vocabulary blocks
  const float* psum;      // partials of rows evaluated again
  int64_t ldp;
  int32_t nmb;
  const int32_t* redo_any;
  int32_t* status;
};

// Per slab token (a wavefront each, two entries a lane): the teacher's entries by ascending id, absent ones
// last (id kAbsent), and, for the logits GEMM, where those of each 256 vocabulary rows begin.  Also no
// sampled token, a cleared shift and flags and, on a call's first slab, the count of rows evaluated again.
__global__ __launch_bounds__(256) void distill_prep_kernel(const DistillParams p, int32_t* __restrict__ yslab,
                                                           float* __restrict__ shift,
                                                           int32_t* __restrict__ flags, int32_t nflags,
                                                           int32_t* __restrict__ count) {
  __shared__ int32_t sorted[4][kMaxDistill];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (first < nflags) flags[first] = 0;
  if (first == 0 && count) count[0] = 0;
  for (int64_t tl = int64_t(blockIdx.x) * 4 + wave; tl < p.Tc; tl += int64_t(gridDim.x) * 4) {
    if (lane == 0) {
      yslab[tl] = -1;
      shift[tl] = 0.0f;
    }
    const int64_t o = (p.t0 + tl) * p.K;
    int y[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k = lane + 64 * u;
      y[u] = k < p.K ? p.ids[o + k] : -1;
      if (y[u] < -1 || y[u] >= p.V) set_status(p.status, FASTRL_SB_BAD_TOKEN);
      if (y[u] < 0 || y[u] >= p.V) y[u] = kAbsent;
    }
    int rank[2] = {0, 0};  // equal ids by entry
    for (int k = 0; k < p.K; ++k) {
      const int yk = __builtin_amdgcn_readlane(k < 64 ? y[0] : y[1], k & 63);
#pragma unroll
      for (int u = 0; u < 2; ++u) rank[u] += yk < y[u] || (yk == y[u] && k < lane + 64 * u);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k = lane + 64 * u;
      if (k < p.K) {
        p.sid[tl * p.K + rank[u]] = y[u];
        p.sa[tl * p.K + rank[u]] = p.a[o + k];
        sorted[wave][rank[u]] = y[u];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (one wavefront writes and reads its row)
    for (int b = lane; b <= p.nmb; b += 64) {
      int lo = 0, hi = p.K;  // ids below 256 b
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sorted[wave][mid] < int64_t(b) * 256) lo = mid + 1;
        else hi = mid;
      }
      p.off[tl * (p.nmb + 1) + b] = uint8_t(lo);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One wavefront per token, two entries a lane.
__device__ __forceinline__ void distill_token(const DistillParams& p, int tl) {
  const int lane = threadIdx.x & 63;
  const int64_t t = p.t0 + tl;
  const float s_t = p.shift[tl];
  const double tau_inv = p.zscale;
  int y[2];
  double x[2], q[2], logq[2], logp[2];
  float z[2];
  bool own[2];  // the first entry of its id
  bool bad = false;
  double m = -INFINITY;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int k = lane + 64 * u;
    y[u] = k < p.K ? p.sid[int64_t(tl) * p.K + k] : kAbsent;
    x[u] = y[u] != kAbsent ? double(p.sa[int64_t(tl) * p.K + k]) : -INFINITY;
    bad |= !(x[u] < INFINITY);
    m = fmax(m, x[u]);
  }
  // (entries lie by id: equal ids side by side)
  auto at = [&](const auto (&v)[2], int pos) {
    const auto lo = __shfl(v[0], pos & 63, 64), hi = __shfl(v[1], pos & 63, 64);
    return pos < 64 ? lo : hi;
  };
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int me = lane + 64 * u, before = at(y, max(me - 1, 0));
    own[u] = y[u] != kAbsent && (me == 0 || before != y[u]);
    z[u] = y[u] != kAbsent ? p.zk[int64_t(tl) * p.K + me] : 0.0f;
  }
  // The student's log-sum-exp from the sum of float32 exponentials (of a row evaluated again: from its
  // new partials).  Their errors grow with z: at z / tau = 60 the exponent alone rounds by 4e-6, and a
  // student close to its teacher has most of the sum in the teacher's entries.  So those are put
  // right: their float32 exponentials, formed here as the GEMM's epilogue does, are replaced.  Without a
  // backward that one forms them relative to the block's maximum, which the merge brings to the token's.
  double S = p.sum[tl], fix = 0.0;
  if (p.E && s_t != 0.0f && p.redo_any[0] != 0) {
    S = 0.0;
    for (int m = lane; m < p.nmb; m += 64) S += double(p.psum[int64_t(m) * p.ldp + tl]);
    S = wave_sum_d(S);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (own[u]) {
      const float ref = p.E ? s_t : p.pmax[int64_t(y[u] >> 8) * p.ldp + tl];
      const float e = p.bf16 ? __builtin_amdgcn_exp2f(fmaf(z[u], 1.4426950408889634f, -(ref * 1.4426950408889634f)))
                             : __expf(z[u] - ref);
      fix += exp(double(z[u]) - double(s_t)) - double(e) * (p.E ? 1.0 : exp(double(ref) - double(s_t)));
    }
  const double l = double(s_t) + log(S + wave_sum_d(fix));
  if (lane == 0) p.lse[t] = float(l);
  double L = 0.0;
  if (p.tlse) {
    L = p.tlse[t];
    bad |= !(fabs(L) < INFINITY);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
  bad = __any(bad);
  const bool some = !bad && m > -INFINITY;  // some entry holds mass
  if (lane == 0 && bad) set_status(p.status, FASTRL_SB_BAD_TEACHER);
  if (!some) {  // contributes nothing
    if (lane == 0) {
      p.token_loss[t] = 0.0f;
      p.term[t] = 0.0;
      p.cslab[tl] = 0.0f;
    }
    return;
  }
  if (!p.tlse) {
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < 2; ++u) s += exp((x[u] - m) * tau_inv);
    L = m * tau_inv + log(wave_sum_d(s));
  }
  double part = 0.0, mass = 0.0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    logq[u] = x[u] * tau_inv - L;
    q[u] = exp(logq[u]);
    logp[u] = double(z[u]) - l;
    mass += q[u];
    if (q[u] > 0.0) part += q[u] * (logq[u] - logp[u]);
  }
  part = wave_sum_d(part);
  mass = wave_sum_d(mass);
  const double w = (p.weight ? double(p.weight[t]) : p.w_default) * p.loss_scale;
  if (lane == 0) {
    p.token_loss[t] = float(part);
    p.term[t] = w * part;
    p.cslab[tl] = float(-w * tau_inv * mass * exp(double(s_t) - l));
  }
  if (!p.E || !(mass > 0.0)) return;
  // an id given more than once: the first takes the others' mass
  double qs[2] = {q[0], q[1]};
  for (int d = 1; d < p.K; ++d) {
    bool any = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int pos = min(lane + 64 * u + d, 127);
      const int yn = at(y, pos);
      const double qn = at(q, pos);
      const bool same = y[u] != kAbsent && lane + 64 * u + d < 128 && yn == y[u];
      if (same) qs[u] += qn;
      any |= same;
    }
    if (!__any(any)) break;
  }
  const double up = exp(l - double(s_t));
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (!own[u]) continue;
    const float e = float((exp(logp[u]) - qs[u] / mass) * up);
    const int64_t o = int64_t(tl) * p.ldE + y[u];
    if (p.bf16) static_cast<uint16_t*>(p.E)[o] = f32_to_bf16(e);
    else static_cast<float*>(p.E)[o] = e;
  }
}

__global__ __launch_bounds__(256) void distill_loss_kernel(const DistillParams p) {
  for (int64_t tl = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); tl < p.Tc; tl += int64_t(gridDim.x) * 4)
    distill_token(p, int(tl));
}

// loss = sum of the tokens' terms in a fixed order: every 1024th to a thread, the threads of a wavefront by butterflies,
// then the wavefronts in order
__global__ __launch_bounds__(1024) void distill_final_kernel(const double* __restrict__ term, int64_t T,
                                                             float* __restrict__ loss) {
  __shared__ double red[16];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < T; i += 1024) s += term[i];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double a = 0.0;
    for (int w = 0; w < 16; ++w) a += red[w];
    loss[0] = float(a);
  }
}

// zeros (dW of a call without tokens)
__global__ __launch_bounds__(256) void distill_zero_kernel(uint16_t* __restrict__ p, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = 0;
}

// bf16 of the float32 dW that several slabs have added up
__global__ __launch_bounds__(256) void distill_round_kernel(const float* __restrict__ in,
                                                            uint16_t* __restrict__ out, int64_t n4) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n4; i += int64_t(gridDim.x) * 256) {
    const f32x4_t v = reinterpret_cast<const f32x4_t*>(in)[i];
    reinterpret_cast<uint2*>(out)[i] = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  }
}

struct DistillWs : LmWs {
  float *sa, *zk, *lse, *token_loss, *dW32;
  int32_t* sid;
  uint8_t* off;
  double* term;
};

// Even shares of at most the asked tokens: slab i is [T i / n, T (i + 1) / n), so of one of two sizes.
struct DistillSlabs {
  int64_t n, size[2];
};

static DistillSlabs distill_slabs(const fastrl_distill_args& a) {
  const int64_t cap = a.slab_tokens > 0 ? a.slab_tokens : kDistillSlab;
  const int64_t n = std::max<int64_t>(1, (a.T + cap - 1) / cap);
  return {n, {a.T / n, (a.T + n - 1) / n}};
}

static LmCall distill_call(const fastrl_distill_args& a, const DistillSlabs& slabs) {
  LmCall c{};
  c.hidden = a.hidden; c.row_index = a.row_index; c.W = a.W;
  c.dtype = a.dtype; c.d = a.d; c.V = a.V; c.T = a.T;
  c.dhidden = a.dhidden; c.dhidden_dtype = a.dhidden_dtype;
  c.dW = a.dW; c.dW_dtype = a.dW_dtype;
  c.tcp = rup(std::max<int64_t>(slabs.size[1], 1), kBN);
  c.zscale = a.temperature == 1.0f ? 0.0f : 1.0f / a.temperature;
  return c;
}

static size_t carve_distill(Carver& c, DistillWs& w, const fastrl_distill_args& a, const LmCall& lc,
                            const DistillSlabs& slabs) {
  const int64_t Vpad = rup(a.V, kBM), tcp = lc.tcp, nmb = Vpad / kBM;
  const int esz = a.dtype == FASTRL_BF16 ? 2 : 4;
  const bool dh = a.dhidden != nullptr, dw = a.dW != nullptr;
  const size_t T = size_t(std::max<int64_t>(a.T, 1));
  const int64_t wt = lm_wt_bytes(lc, slabs.size, 2);
  w.WT = wt > 0 ? c.take<char>(size_t(wt)) : nullptr;
  w.E1 = (dh || dw) ? c.take<char>(size_t(tcp) * Vpad * esz) : nullptr;
  w.Bd = dw ? c.take<char>(size_t(a.d) * tcp * esz) : nullptr;
  w.dW32 = dw && a.dW_dtype == FASTRL_BF16 && slabs.n > 1 ? c.take<float>(size_t(a.V) * a.d) : nullptr;
  w.pmax = c.take<float>(size_t(nmb * tcp));
  w.psum = c.take<float>(size_t(nmb * tcp));
  w.psz = nullptr;
  w.zlab = c.take<float>(size_t(tcp));
  w.shift = c.take<float>(size_t(tcp));
  w.cslab = c.take<float>(size_t(tcp));
  w.yslab = c.take<int32_t>(size_t(tcp));
  w.redo_blk = c.take<int32_t>(size_t(tcp / kBN + 1));
  w.redo_count = c.take<int32_t>(1);
  w.sid = c.take<int32_t>(size_t(tcp) * a.K);
  w.sa = c.take<float>(size_t(tcp) * a.K);
  w.zk = c.take<float>(size_t(tcp) * a.K);
  w.off = c.take<uint8_t>(size_t(tcp) * size_t(nmb + 1));
  w.sum = c.take<float>(size_t(tcp));
  w.pick_ids = w.sid; w.pick_off = w.off; w.pick_z = w.zk;
  w.pick_n = a.K; w.pick_ldo = int32_t(nmb + 1);
  w.lse = a.lse ? a.lse : c.take<float>(T);
  w.token_loss = a.token_loss ? a.token_loss : c.take<float>(T);
  w.term = c.take<double>(T);
  return c.size();
}

// blocks of four wavefronts for n items, each wavefront taking several where a launch cannot hold them
static unsigned wave_blocks(int64_t n) {
  return unsigned(std::min<int64_t>((n + 3) / 4, 4 * kMaxBlocks));
}

static int run_distill(const fastrl_distill_args& a, hipStream_t stream) {
  const DistillSlabs slabs = distill_slabs(a);
  LmCall lc = distill_call(a, slabs);
  Carver c(a.ws);
  DistillWs w;
  carve_distill(c, w, a, lc, slabs);
  const bool dw = a.dW != nullptr, store = a.dhidden || dw;
  const int64_t nW = int64_t(a.V) * a.d;
  if (a.T == 0 && dw && !a.dW_accumulate) {
    hipLaunchKernelGGL(distill_zero_kernel, dim3(1024), dim3(256), 0, stream,
                       static_cast<uint16_t*>(a.dW), a.dW_dtype == FASTRL_BF16 ? nW : 2 * nW);
    FR_LAUNCHED();
  }
  if (w.dW32) {
    lc.dW = w.dW32;
    lc.dW_dtype = FASTRL_F32;
  }
  if (a.T > 0) FR_TRY(lm_prepare(lc, w, stream));
  DistillParams p{};
  p.V = a.V; p.K = a.K;
  p.ids = a.top_ids; p.a = a.top_logits; p.tlse = a.teacher_lse; p.weight = a.weight;
  p.w_default = a.T > 0 ? 1.0 / double(a.T) : 0.0; p.loss_scale = a.loss_scale;
  p.zscale = 1.0f / a.temperature;
  p.sid = w.sid; p.sa = w.sa; p.off = w.off; p.zk = w.zk; p.lse = w.lse; p.token_loss = w.token_loss; p.term = w.term; p.cslab = w.cslab;
  p.E = store ? w.E1 : nullptr; p.ldE = rup(a.V, kBM); p.bf16 = a.dtype == FASTRL_BF16;
  p.shift = w.shift; p.sum = w.sum; p.pmax = w.pmax; p.psum = w.psum; p.ldp = lc.tcp;
  p.nmb = int32_t(rup(a.V, kBM) / kBM); p.status = a.status;
  for (int64_t i = 0; i < slabs.n && a.T > 0; ++i) {
    const int64_t t0 = a.T * i / slabs.n;
    const int32_t Tc = int32_t(a.T * (i + 1) / slabs.n - t0);
    const int32_t nnb = int32_t(rup(Tc, kBN) / kBN);
    p.t0 = t0; p.Tc = Tc; p.redo_any = lm_redo_any(w, Tc);
    // (nnb + 1 flags: at least one block of 256 threads, and four tokens a block)
    hipLaunchKernelGGL(distill_prep_kernel, dim3(wave_blocks(Tc)), dim3(256), 0, stream, p, w.yslab,
                       w.shift, w.redo_blk, nnb + 1, i == 0 ? w.redo_count : (int32_t*)nullptr);
    FR_LAUNCHED();
    FR_TRY(lm_forward(lc, w, t0, Tc, w.lse, nullptr, nullptr, stream));
    hipLaunchKernelGGL(distill_loss_kernel, dim3(wave_blocks(Tc)), dim3(256), 0, stream, p);
    FR_LAUNCHED();
    FR_TRY(lm_backward(lc, w, t0, Tc, i > 0 || a.dW_accumulate, stream));
  }
  if (w.dW32 && a.T > 0) {
    hipLaunchKernelGGL(distill_round_kernel, dim3(4096), dim3(256), 0, stream, w.dW32,
                       static_cast<uint16_t*>(a.dW), nW / 4);
    FR_LAUNCHED();
  }
  hipLaunchKernelGGL(distill_final_kernel, dim3(1), dim3(1024), 0, stream, w.term, a.T, a.loss);
  FR_LAUNCHED();
  return FASTRL_OK;
}

static int check_distill_args(const fastrl_distill_args* a, bool need_ws) {
  const std::string f = "fastrl_distill_loss";
  FR_CHECK_ARG(a != nullptr, FASTRL_ERR_NULL_PTR, f + ": args is NULL");
  auto dtype_ok = [](int32_t t) { return t == FASTRL_F32 || t == FASTRL_BF16; };
  FR_CHECK_ARG(dtype_ok(a->dtype), FASTRL_ERR_DTYPE, f + ": dtype must be FASTRL_F32 or FASTRL_BF16");
  FR_CHECK_ARG(!a->dhidden || dtype_ok(a->dhidden_dtype), FASTRL_ERR_DTYPE, f + ": bad dhidden_dtype");
  FR_CHECK_ARG(!a->dW || dtype_ok(a->dW_dtype), FASTRL_ERR_DTYPE, f + ": bad dW_dtype");
  FR_CHECK_ARG(!a->dW || a->dW_dtype == FASTRL_F32 || (a->dtype == FASTRL_BF16 && !a->dW_accumulate),
               FASTRL_ERR_UNSUPPORTED,
               f + ": a bfloat16 dW needs bfloat16 operands and cannot be accumulated into");
  FR_CHECK_ARG(a->d >= 8 && a->d % 8 == 0 && a->V >= 1 && a->V < (1 << 30) && a->T >= 0 &&
                   a->T < (int64_t(1) << 31),
               FASTRL_ERR_SHAPE, f + ": need d a positive multiple of 8, 1 <= V < 2^30, 0 <= T < 2^31");
  FR_CHECK_ARG(a->K >= 1 && a->K <= kMaxDistill, FASTRL_ERR_SHAPE, f + ": K must be in [1, 128]");
  FR_CHECK_ARG(std::isfinite(a->temperature) && a->temperature > 0.0f &&
                   std::isfinite(1.0f / a->temperature),
               FASTRL_ERR_VALUE, f + ": temperature must be finite and > 0");
  FR_CHECK_ARG(std::isfinite(a->loss_scale), FASTRL_ERR_VALUE, f + ": loss_scale not finite");
  FR_CHECK_ARG(a->slab_tokens >= 0, FASTRL_ERR_VALUE, f + ": slab_tokens < 0");
  FR_CHECK_ARG(a->loss, FASTRL_ERR_NULL_PTR, f + ": loss is NULL");
  auto al = [](const void* x, uintptr_t n) { return (reinterpret_cast<uintptr_t>(x) % n) == 0; };
  if (a->T > 0) {
    FR_CHECK_ARG(a->hidden && a->W && a->top_ids && a->top_logits, FASTRL_ERR_NULL_PTR,
                 f + ": hidden / W / top_ids / top_logits is NULL");
    FR_CHECK_ARG(al(a->hidden, 16) && al(a->W, 16) && al(a->dW, 16), FASTRL_ERR_VALUE,
                 f + ": hidden, W and dW must be 16-byte aligned");
  }
  if (need_ws) {
    const size_t need = fastrl_distill_loss_workspace_size(a);
    FR_CHECK_ARG(a->ws && al(a->ws, 256) && a->ws_bytes >= need, FASTRL_ERR_WORKSPACE,
                 f + ": workspace missing, misaligned or smaller than " + std::to_string(need) + " bytes");
  }
  return FASTRL_OK;
}

}  // namespace fastrl

using namespace fastrl;

extern "C" {

size_t fastrl_distill_args_size(void) { return sizeof(fastrl_distill_args); }

size_t fastrl_distill_loss_workspace_size(const fastrl_distill_args* args) {
  clear_error();
  if (check_distill_args(args, false) != FASTRL_OK) return 0;
  const DistillSlabs slabs = distill_slabs(*args);
  Carver c(nullptr);
  DistillWs w;
  return carve_distill(c, w, *args, distill_call(*args, slabs), slabs);
}

int fastrl_distill_loss_fwd_bwd(const fastrl_distill_args* args, hipStream_t stream) {
  clear_error();
  const int rc = check_distill_args(args, true);
  if (rc != FASTRL_OK) return rc;
  return run_distill(*args, stream);
}

}  // extern "C"
