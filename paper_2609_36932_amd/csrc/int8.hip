// Rows of activations or weights to int8 codes with a scale each, and products of such codes.
//
//   m_t = max_k |x[t,k]|,  s_t = m_t / 127,  q[t,k] = rint(x[t,k] * (127 / m_t))
//   out[t,n] = float(sum_k q[t,k] w[n,k]) * s_t * c_n
//
// The sum is an exact 32-bit integer, so it does not depend on the order, the tiling or the number of
// tokens beside it; the two float32 products are made in the order written.
#include <string>

#include "gemm_loop.h"
#include "int8.h"

namespace fastrl {

// 16 bytes of rows of any width
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_u __attribute__((ext_vector_type(4), aligned(2)));

// ------------------------------------------------------------------ codes

// rows whose largest entry is below this count as rows of zeros (127 / m would leave float range
// at 2^-121)
constexpr float kTinyRow = 7.888609052210118e-31f;  // 2^-100
constexpr int kQuantThreads = 256;

// bits of columns k .. k + 7 of a row as float32 (0 past its end); rows need no alignment: global memory
// takes 16-byte accesses at any element
template <typename T>
__device__ __forceinline__ void row_piece(const T* row, int64_t k, int32_t K, uint32_t (&v)[8]) {
  if (k + 8 <= K) {
    if constexpr (sizeof(T) == 2) {
      const u32x4_t r = *reinterpret_cast<const u32x4_u*>(row + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = r[e] << 16;
        v[2 * e + 1] = r[e] & 0xffff0000u;
      }
    } else {
      const u32x4_t a = *reinterpret_cast<const u32x4_u*>(row + k);
      const u32x4_t b = *reinterpret_cast<const u32x4_u*>(row + k + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = a[e];
        v[4 + e] = b[e];
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0;
      if (k + e < K) {
        if constexpr (sizeof(T) == 2) v[e] = uint32_t(row[k + e]) << 16;
        else v[e] = __float_as_uint(row[k + e]);
      }
    }
  }
}

// maximum of |x| on the bits: as integers they order like the numbers, with infinities and NaN above them
__device__ __forceinline__ uint32_t piece_peak(uint32_t m, const uint32_t (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, v[e] & 0x7fffffffu);
  return m;
}

struct RowScale {
  float inv, scale;
  bool some;  // else every code is 0 (a row that is not finite would leave NaN * 0)
};
__device__ __forceinline__ RowScale row_scale(uint32_t peak) {
  const float amax = __uint_as_float(peak);
  const bool finite = peak < 0x7f800000u, some = finite && amax >= kTinyRow;
  return {some ? 127.0f / amax : 0.0f, some ? amax / 127.0f : finite ? 0.0f : __int_as_float(0x7fc00000), some};
}

__device__ __forceinline__ uint2 piece_codes(const RowScale& s, const uint32_t (&v)[8]) {
  uint32_t b[2] = {0, 0};
  if (s.some)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      b[e >> 2] |= (uint32_t(int(rintf(__uint_as_float(v[e]) * s.inv))) & 0xffu) << (8 * (e & 3));
  return make_uint2(b[0], b[1]);
}

// codes of columns k .. k + 7, and zeros up to the end of the output row
__device__ __forceinline__ void store_codes(int8_t* out, int64_t k, int64_t ldq, const RowScale& s,
                                            const uint32_t (&v)[8]) {
  const uint2 b = piece_codes(s, v);
  if (k + 8 <= ldq && ((reinterpret_cast<uintptr_t>(out) + k) & 7) == 0) {
    *reinterpret_cast<uint2*>(out + k) = b;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < ldq) out[k + e] = int8_t((e < 4 ? b.x : b.y) >> (8 * (e & 3)));
  }
}

// One block per row: bound by latency, reading the row and exchanging the maximum.  A thread keeps PIECES pieces of
// 8 columns in registers between maximum and codes; what a longer row has beyond is read again (from L2).
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(
    const T* __restrict__ x, const int32_t* __restrict__ row_index, int32_t K, int64_t ldx,
    int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, int64_t row0) {
  constexpr int PIECES = 2;
  __shared__ uint32_t red[kQuantThreads / 64];
  const int64_t t = row0 + blockIdx.x;
  const T* row = x + int64_t(row_index ? row_index[t] : t) * ldx;
  uint32_t keep[PIECES][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) row_piece(row, (int64_t(i) * kQuantThreads + threadIdx.x) * 8, K, keep[i]);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) m = piece_peak(m, keep[i]);
  const int64_t beyond = int64_t(PIECES) * kQuantThreads * 8;
  for (int64_t k = beyond + threadIdx.x * 8; k < K; k += kQuantThreads * 8) {
    uint32_t v[8];
    row_piece(row, k, K, v);
    m = piece_peak(m, v);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, 64)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / 64; ++w) m = max(m, red[w]);
  const RowScale s = row_scale(m);
  if (threadIdx.x == 0) scale[t] = s.scale;
  int8_t* out = q + t * ldq;
#pragma unroll
  for (int i = 0; i < PIECES; ++i)
    store_codes(out, (int64_t(i) * kQuantThreads + threadIdx.x) * 8, ldq, s, keep[i]);
  for (int64_t k = beyond + threadIdx.x * 8; k < ldq; k += kQuantThreads * 8) {
    uint32_t v[8];
    row_piece(row, k, K, v);
    store_codes(out, k, ldq, s, v);
  }
}

// One wavefront per row of at most 512 PIECES columns, all of it in registers
template <typename T, int PIECES>
__global__ __launch_bounds__(kQuantThreads) void quantize_wave_kernel(
    const T* __restrict__ x, const int32_t* __restrict__ row_index, int32_t K, int64_t ldx,
    int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, int64_t row0, int64_t rows) {
  const int lane = threadIdx.x & 63;
  const int64_t t = row0 + int64_t(blockIdx.x) * (kQuantThreads / 64) + (threadIdx.x >> 6);
  if (t >= rows) return;
  const T* row = x + int64_t(row_index ? row_index[t] : t) * ldx;
  uint32_t keep[PIECES][8];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) row_piece(row, (64 * i + lane) * 8, K, keep[i]);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) m = piece_peak(m, keep[i]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, 64)));
  const RowScale s = row_scale(m);
  if (lane == 0) scale[t] = s.scale;
  int8_t* out = q + t * ldq;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) store_codes(out, (64 * i + lane) * 8, ldq, s, keep[i]);
}

template <typename T>
static int launch_quantize_rows(const T* x, const int32_t* row_index, int64_t rows, int32_t K, int64_t ldx, int8_t* q,
                                int64_t ldq, float* scale, hipStream_t stream) {
  // us, a block / a wavefront per row: 8191 rows of 557 22.6 / 7.6, of 1536 19.0 / 14.5, of 3584 18.8 / 19.3 (4.7 TB/s
  // of reads and writes, most from caches); 600 of 1536 4.4 / 4.0, of 3584 4.2 / 5.6; 193 of 1536 3.9 / 4.0
  const bool wave = ldq <= 1024 || (ldq <= 2048 && rows >= 512);
  const int64_t per = wave ? kQuantThreads / 64 : 1;
  for (int64_t t = 0; t < rows; t += per * kMaxBlocks) {
    const dim3 grid(unsigned(std::min((rows - t + per - 1) / per, kMaxBlocks))), block(kQuantThreads);
    if (wave) {
      const auto f = ldq <= 512    ? quantize_wave_kernel<T, 1>
                     : ldq <= 1024 ? quantize_wave_kernel<T, 2>
                                   : quantize_wave_kernel<T, 4>;
      hipLaunchKernelGGL(f, grid, block, 0, stream, x, row_index, K, ldx, q, ldq, scale, t, rows);
    } else {
      hipLaunchKernelGGL(quantize_kernel<T>, grid, block, 0, stream, x, row_index, K, ldx, q, ldq, scale, t);
    }
    FR_LAUNCHED();
  }
  return FASTRL_OK;
}

int launch_quantize(const void* x, int32_t dtype, const int32_t* row_index, int64_t T, int32_t K,
                    int64_t ldx, int8_t* q, int64_t ldq, float* scale, hipStream_t stream) {
  if (dtype == FASTRL_BF16)
    return launch_quantize_rows(static_cast<const uint16_t*>(x), row_index, T, K, ldx, q, ldq, scale, stream);
  return launch_quantize_rows(static_cast<const float*>(x), row_index, T, K, ldx, q, ldq, scale, stream);
}

// ------------------------------------------------------------------ product

constexpr int kGroup = 32;  // channel blocks of a sweep over the tokens

struct I8Params : GemmParams {
  const float *xs, *ws;
  void* out;
  int64_t ldo;
  int32_t out_bf16;
  int32_t staged;  // output rows do not all start at 16 bytes (store_rows)
  int32_t width;   // tokens of a tile column: 64 to 256
  int32_t whole;   // tiles before the cut ones
  int32_t pieces;  // blocks of a cut tile
  float2* part;
  int64_t ldpart;
  uint32_t* mask;
  const float* bound;
  float tau2;      // log2(e) / tau
};

// 16 bytes from byte `a` (0 to 15, even) of the 32 bytes lo, hi
__device__ __forceinline__ u32x4_t bytes_from(u32x4_t lo, u32x4_t hi, int a) {
  const bool s2 = a & 8, s1 = a & 4;
  const uint32_t c0 = s2 ? lo[2] : lo[0], c1 = s2 ? lo[3] : lo[1], c2 = s2 ? hi[0] : lo[2],
                 c3 = s2 ? hi[1] : lo[3], c4 = s2 ? hi[2] : hi[0], c5 = s2 ? hi[3] : hi[1];
  const uint32_t d0 = s1 ? c1 : c0, d1 = s1 ? c2 : c1, d2 = s1 ? c3 : c2, d3 = s1 ? c4 : c3, d4 = s1 ? c5 : c4;
  const uint32_t by = a & 3;
  return u32x4_t{__builtin_amdgcn_alignbyte(d1, d0, by), __builtin_amdgcn_alignbyte(d2, d1, by),
                 __builtin_amdgcn_alignbyte(d3, d2, by), __builtin_amdgcn_alignbyte(d4, d3, by)};
}

// Output rows that do not start at 16 bytes: a wavefront's 16 tokens x 128 channels lie in its part of LDS as
// token rows (a 16-byte chunk longer than they are, so that rows begin in different banks) and go out as whole
// aligned 16-byte chunks, neighbouring lanes writing neighbouring ones, and up to 15 bytes before and after
// them element by element.  Stored straight from the registers, each quad of channels wrote parts of two
// chunks: 2433 x 640 x 78593 (T x K x N) 353 us in float32 and 325 in bf16, so 328 and 251 (N = 78592: 263 and 197;
// what is left are lines that two blocks write parts of).
constexpr int kRowStage = 20480;  // bytes of a wavefront's part
template <int ESZ>
__device__ __forceinline__ void store_rows(const I8Params& p, const char* rows, int t0, int v0, int lane) {
  constexpr int CH = 128 * ESZ / 16, PITCH = 16 * (CH + 1), PER = 64 / CH;  // chunks of a row; rows of a store
  const int bytes = min(128, p.M - v0) * ESZ;
  auto to = [&](int r) {
    return static_cast<char*>(p.out) + (int64_t(t0 + r) * p.ldo + v0) * ESZ;
  };
#pragma unroll
  for (int r0 = 0; r0 < 16; r0 += PER) {
    const int r = r0 + lane / CH, l = lane % CH;
    char* o = to(r);
    const int a = int(-reinterpret_cast<uintptr_t>(o) & 15);
    const u32x4_t* c = reinterpret_cast<const u32x4_t*>(rows + r * PITCH) + l;
    const u32x4_t x = bytes_from(c[0], c[1], a);
    if (t0 + r < p.N && a + 16 * l + 16 <= bytes) *reinterpret_cast<u32x4_t*>(o + a + 16 * l) = x;
  }
  const int r = lane & 15;
  char* o = to(r);
  const int a = int(-reinterpret_cast<uintptr_t>(o) & 15), first = min(a, bytes);
  const int last = bytes > a ? a + ((bytes - a) & ~15) : bytes;
  if (t0 + r >= p.N) return;
#pragma unroll
  for (int e0 = 0; e0 < 16 / ESZ; e0 += 4) {
    const int e = (e0 + (lane >> 4)) * ESZ;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = h ? last + e : e;
      if (b < (h ? bytes : first)) {
        const uint32_t x = *reinterpret_cast<const uint32_t*>(rows + r * PITCH + (b & ~3));
        if constexpr (ESZ == 4) *reinterpret_cast<uint32_t*>(o + b) = x;
        else *reinterpret_cast<uint16_t*>(o + b) = uint16_t(x >> (8 * (b & 2)));
      }
    }
  }
}

// Epilogue: acc[i][j][q] is the sum of output channel v = m0 + wm*128 + 16 i + 4 (l / 16) + q and token
// n0 + wn*16 NJ + 16 j + l % 16, so a lane's four are neighbours in the token's output row.  FULL: all
// 256 channels exist, and output rows start at 16 bytes.
template <int NJ, bool FULL, bool PART>
__device__ __forceinline__ void i8_epilogue(const I8Params& p, int m0, int n0, i32x4_t (&acc)[8][NJ],
                                            uint16_t* smem) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 2, wn = wave & 3, g = lane >> 4, c = lane & 15;
  const int v0 = m0 + wm * 128 + 4 * g;
  char* const stage = reinterpret_cast<char*>(smem) + wave * kRowStage;
  if (!PART && !FULL && p.staged) __syncthreads();  // no wavefront reads the operands any more
  f32x4_t ws[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (FULL) {
      ws[i] = *reinterpret_cast<const f32x4_u*>(p.ws + v0 + 16 * i);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) ws[i][q] = p.ws[min(v0 + 16 * i + q, p.M - 1)];
    }
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int t = n0 + wn * 16 * NJ + 16 * j + c;
    const bool ok = t < p.N;
    const float s = ok ? p.xs[t] : 0.0f;
    f32x4_t z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) z[i][q] = float(acc[i][j][q]) * s * ws[i][q];
    if constexpr (PART) {
      // group's maximum, sum and, written as whole quads, the logits that can be among the largest
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, sm[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const float bound = p.bound && ok ? p.bound[t] : -INFINITY;
      float* o = static_cast<float*>(p.out) + int64_t(t) * p.ldo;
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int v = v0 + 16 * i;
        float qm = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (FULL || v + q < p.M) qm = fmaxf(qm, z[i][q]);
        mx[i & 3] = fmaxf(mx[i & 3], qm);
        if (ok && (FULL || v < p.M) && qm >= bound) {
          *reinterpret_cast<f32x4_t*>(o + v) = z[i];
          bits |= 1u << (4 * i);
        }
      }
      const float m = group_max4(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
      const float ml = m > -INFINITY ? m * p.tau2 : 0.0f;  // (a group of -infinity alone has the sum 0)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (FULL || v0 + 16 * i + q < p.M)
            sm[i & 3] += __builtin_amdgcn_exp2f(fmaf(z[i][q], p.tau2, -ml));
      const float sum = group_sum4((sm[0] + sm[1]) + (sm[2] + sm[3]));
      bits = group_or4(bits << g);
      if (g == 0 && ok && m0 + wm * 128 < p.M) {
        const int64_t e = int64_t(t) * p.ldpart + (m0 + wm * 128) / kTopkGroup;
        p.part[e] = make_float2(m, sum);
        p.mask[e] = bits;
      }
    } else if (!FULL && p.staged) {
      if (p.out_bf16) {
        char* row = stage + c * 272 + 8 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<uint2*>(row + 32 * i) =
              make_uint2(pack_bf16(z[i][0], z[i][1]), pack_bf16(z[i][2], z[i][3]));
      } else {
        char* row = stage + c * 528 + 16 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<f32x4_t*>(row + 64 * i) = z[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wavefront's own rows)
      if (p.out_bf16) store_rows<2>(p, stage, t - c, m0 + wm * 128, lane);
      else store_rows<4>(p, stage, t - c, m0 + wm * 128, lane);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else if (p.out_bf16) {
      uint16_t* o = static_cast<uint16_t*>(p.out) + int64_t(t) * p.ldo;
#pragma unroll
      for (int ip = 0; ip < 4; ++ip) {  // 8 neighbours a lane: rows swapped between lane groups
        uint32_t pk[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          pk[h][0] = pack_bf16(z[2 * ip + h][0], z[2 * ip + h][1]);
          pk[h][1] = pack_bf16(z[2 * ip + h][2], z[2 * ip + h][3]);
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const auto sw = __builtin_amdgcn_permlane16_swap(pk[0][w], pk[1][w], false, false);
          pk[0][w] = sw[0];
          pk[1][w] = sw[1];
        }
        const int v = m0 + wm * 128 + (2 * ip + (g & 1)) * 16 + (g >> 1) * 8;
        const u32x4_t r = {pk[0][0], pk[0][1], pk[1][0], pk[1][1]};
        if (ok && (FULL || v + 8 <= p.M)) {
          *reinterpret_cast<u32x4_u*>(o + v) = r;
        } else if (ok) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (v + q < p.M) o[v + q] = uint16_t(r[q >> 1] >> (16 * (q & 1)));
        }
      }
    } else if (ok) {
      float* o = static_cast<float*>(p.out) + int64_t(t) * p.ldo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int v = v0 + 16 * i;
        if (FULL || v + 4 <= p.M) {
          *reinterpret_cast<f32x4_u*>(o + v) = z[i];
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (v + q < p.M) o[v + q] = z[i][q];
        }
      }
    }
  }
}

template <int NJ, bool PART>
__device__ __forceinline__ void i8_tile(const I8Params& p, int mb, int n0, uint16_t* smem) {
  i32x4_t acc[8][NJ];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  mfma_mainloop<MODE_FWD, NJ>(p, mb * kBM, n0, acc, smem);
  if ((mb + 1) * kBM <= p.M && (PART || !p.staged)) i8_epilogue<NJ, true, PART>(p, mb * kBM, n0, acc, smem);
  else i8_epilogue<NJ, false, PART>(p, mb * kBM, n0, acc, smem);
}

// The matrix product of many tokens, on the main loop of the bf16 GEMMs (gemm_loop.h) with its 16-byte pieces
// read as 16 codes: 2,640 TOP/s at 16384^3 (bf16 1,564 by the vendor's library, int8 2,265), 2,410 in the product
// of 8191 tokens at 7B, whose 28 K steps a tile bear a start and an epilogue of ~8 us.  Blocks that walk several
// tiles and load the next one's first stages during the epilogue measured 5% slower (in a form that waited for
// the stores, and spilled); two blocks a compute unit, of 128 channels x 192 tokens in two stages of 40 KB each, took 12% less
// time at K = 320 (2433 x 78592 products in bf16: 171 / 150 us), 6% less at 640, 6% more at 1536 and 15% at 3584: not
// kept, a main loop of its own for K below about 1000 alone.
// Tiles of 256 output channels x `width` tokens, the last column as narrow as its tokens allow; the last tiles,
// which do not fill the chip, cut into pieces of fewer tokens (tile_plan).
template <bool PART>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void i8_gemm_kernel(const I8Params p) {
  __shared__ __attribute__((aligned(1024))) char smem_raw[kSmemBytes];
  uint16_t* smem = reinterpret_cast<uint16_t*>(smem_raw);
  int b = p.block0 + int(blockIdx.x), piece = 0, pieces = 1;
  if (b >= p.whole) {
    // the pieces of a tile 8 blocks apart, and so on one XCD: they read the same codes of the weight
    pieces = p.pieces;
    const int i = b - p.whole, g = i / (8 * pieces);
    piece = (i >> 3) % pieces;
    b = p.whole + 8 * g + (i & 7);
    if (b >= p.nmb * p.nnb) return;
  }
  int mb, nb;
  tile_coords<MODE_FWD>(mb, nb, p.nmb, p.nnb, b, p.group);
  // (a full group's blocks are dealt to the 8 XCDs in turn: neighbours go to one of them, whose cache then joins
  // the lines that both write parts of)
  const int in = mb % kGroup;
  if (p.staged && mb - in + kGroup <= p.nmb) mb += (in & 7) * (kGroup / 8) + (in >> 3) - in;
  int n0 = nb * p.width;
  int cols = (min(p.width, p.N - n0) + 63) >> 6;
  if (pieces > 1) {
    const int per = (cols + pieces - 1) / pieces;
    n0 += piece * per * 64;
    cols = min(per, cols - piece * per);
    if (cols <= 0) return;
  }
  if (cols == 4) i8_tile<4, PART>(p, mb, n0, smem);
  else if (cols == 3) i8_tile<3, PART>(p, mb, n0, smem);
  else if (cols == 2) i8_tile<2, PART>(p, mb, n0, smem);
  else i8_tile<1, PART>(p, mb, n0, smem);
}

// Few tokens and output channels: whole tiles would leave most compute units idle, so a block takes
// only 16 MR channels and 16 NT tokens, and its eight wavefronts share K, 64 columns in turn, each with the
// next step's codes in flight while it multiplies the present ones.  The eight sums meet in LDS (integers:
// any order gives the same); wavefront w finishes tile w.
template <int NT, int MR>
__global__ __launch_bounds__(512) void i8_skinny_kernel(const I8Params p) {
  constexpr int W = 8;
  __shared__ i32x4_t part[W][MR][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  // blocks are dealt to the 8 XCDs in turn: those that read the same codes of the weight go to one of them, one
  // after the other; fewer than 8 such sets are dealt over all of them
  const int id = p.block0 + int(blockIdx.x);
  const bool few = p.nmb < 8;
  const int mb = few ? id % p.nmb : id / (8 * p.nnb) * 8 + (id & 7);
  const int n0 = (few ? id / p.nmb : (id >> 3) % p.nnb) * 16 * NT;
  const int m0 = mb * 16 * MR;
  if (mb >= p.nmb) return;
  const char* const A = static_cast<const char*>(p.A);
  const char* const B = static_cast<const char*>(p.B);
  const char* ap[MR];
  const char* bp[NT];
#pragma unroll
  for (int i = 0; i < MR; ++i) ap[i] = A + 2 * int64_t(min(m0 + 16 * i + c, p.M - 1)) * p.lda;
#pragma unroll
  for (int j = 0; j < NT; ++j) bp[j] = B + 2 * int64_t(min(n0 + 16 * j + c, p.N - 1)) * p.ldb;
  const int K = 2 * p.K, ns = (K + 63) / 64;
  i32x4_t acc[MR][NT];
#pragma unroll
  for (int i = 0; i < MR; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  i32x4_t a[2][MR], b[2][NT];
  auto load = [&](int s, i32x4_t (&fa)[MR], i32x4_t (&fb)[NT]) {
    const int k = min(64 * s + 16 * g, K - 16);  // (pieces past K load a valid one, and count as 0)
    const bool past = 64 * s + 16 * g >= K;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      fb[j] = *reinterpret_cast<const i32x4_t*>(bp[j] + k);
      if (past) fb[j] = i32x4_t{0, 0, 0, 0};
    }
    // (not past the caches: two wavefronts read the halves of a line)
#pragma unroll
    for (int i = 0; i < MR; ++i) fa[i] = *reinterpret_cast<const i32x4_t*>(ap[i] + k);
  };
  auto multiply = [&](const i32x4_t (&fa)[MR], const i32x4_t (&fb)[NT]) {
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
  };
  int s = wave;
  if (s < ns) load(s, a[0], b[0]);
  for (; s < ns; s += 2 * W) {
    if (s + W < ns) load(s + W, a[1], b[1]);
    multiply(a[0], b[0]);
    if (s + W < ns) {
      if (s + 2 * W < ns) load(s + 2 * W, a[0], b[0]);
      multiply(a[1], b[1]);
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    if (j > 0) __syncthreads();  // the sums of the tokens before are read
#pragma unroll
    for (int i = 0; i < MR; ++i) part[wave][i][lane] = acc[i][j];
    __syncthreads();
    const int t = n0 + 16 * j + c;
    if (wave < MR && t < p.N) {
      i32x4_t sum = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < W; ++w) sum += part[w][wave][lane];
      const float sx = p.xs[t];
      const int v = m0 + 16 * wave + 4 * g;
      f32x4_t z;
#pragma unroll
      for (int q = 0; q < 4; ++q) z[q] = float(sum[q]) * sx * p.ws[min(v + q, p.M - 1)];
      const bool whole = v + 4 <= p.M;
      if (p.out_bf16) {
        uint16_t* o = static_cast<uint16_t*>(p.out) + int64_t(t) * p.ldo + v;
        typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(2)));
        if (whole) {
          *reinterpret_cast<u32x2_u*>(o) = u32x2_u{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3])};
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (v + q < p.M) o[q] = f32_to_bf16(z[q]);
        }
      } else {
        float* o = static_cast<float*>(p.out) + int64_t(t) * p.ldo + v;
        if (whole) {
          *reinterpret_cast<f32x4_u*>(o) = z;
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (v + q < p.M) o[q] = z[q];
        }
      }
    }
  }
}

// One to sixteen tokens and few channels, in one launch: every block codes the rows itself (into LDS, while its
// first codes of the weight are on their way) and goes on like i8_skinny_kernel<1, 1>.  Up to four tokens: the
// whole block codes a row at a time; more: each wavefront two rows of its own.
// bytes of codes in LDS, without the rows' ends
constexpr int token_codes(int tok) { return tok > 4 ? 57344 : 32768; }
template <typename T, int TOK>
__global__ __launch_bounds__(512) void i8_token_kernel(const I8Params p, const T* __restrict__ x,
                                                       const int32_t* __restrict__ row_index, int64_t ldx,
                                                       int32_t Kx) {
  constexpr int W = 8;
  constexpr bool OWN = TOK > 4;  // a wavefront's rows are its own
  constexpr int KEEP = OWN ? 4 : TOK;
  __shared__ __attribute__((aligned(16))) int8_t codes[token_codes(TOK) + 16 * TOK];
  __shared__ i32x4_t part[W][64];
  __shared__ uint32_t red[W][TOK];
  __shared__ float xs[TOK];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int m0 = blockIdx.x * 16;
  const int K = 2 * p.K, ns = (K + 63) / 64;
  const int pitch = K | 16;  // (rows begin in different banks)
  const char* const A = static_cast<const char*>(p.A) + 2 * int64_t(min(m0 + c, p.M - 1)) * p.lda;
  // (pieces past K load a valid one, and count as 0)
  auto weight = [&](int s) { return *reinterpret_cast<const i32x4_t*>(A + min(64 * s + 16 * g, K - 16)); };
  auto source = [&](int t) { return x + int64_t(row_index ? row_index[t] : t) * ldx; };
  i32x4_t a[2];
  if (wave < ns) a[0] = weight(wave);
  if (wave + W < ns) a[1] = weight(wave + W);
  uint32_t keep[KEEP][8];
  if constexpr (OWN) {
    for (int t = wave; t < p.N; t += W) {
      const T* row = source(t);
#pragma unroll
      for (int i = 0; i < KEEP; ++i) row_piece(row, (64 * i + lane) * 8, Kx, keep[i]);
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < KEEP; ++i) m = piece_peak(m, keep[i]);
      for (int k = (64 * KEEP + lane) * 8; k < Kx; k += 512) {
        uint32_t v[8];
        row_piece(row, k, Kx, v);
        m = piece_peak(m, v);
      }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, 64)));
      const RowScale s = row_scale(m);
      if (lane == 0) xs[t] = s.scale;
#pragma unroll
      for (int i = 0; i < KEEP; ++i) {
        const int k = (64 * i + lane) * 8;
        if (k < K) *reinterpret_cast<uint2*>(codes + t * pitch + k) = piece_codes(s, keep[i]);
      }
      for (int k = (64 * KEEP + lane) * 8; k < K; k += 512) {
        uint32_t v[8];
        row_piece(row, k, Kx, v);
        *reinterpret_cast<uint2*>(codes + t * pitch + k) = piece_codes(s, v);
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < TOK; ++t) {
      if (t >= p.N) break;
      const T* row = source(t);
      row_piece(row, threadIdx.x * 8, Kx, keep[t]);
      uint32_t m = piece_peak(0, keep[t]);
      for (int k = (512 + threadIdx.x) * 8; k < Kx; k += 512 * 8) {
        uint32_t v[8];
        row_piece(row, k, Kx, v);
        m = piece_peak(m, v);
      }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, 64)));
      if (lane == 0) red[wave][t] = m;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TOK; ++t) {
      if (t >= p.N) break;
      uint32_t m = red[0][t];
#pragma unroll
      for (int w = 1; w < W; ++w) m = max(m, red[w][t]);
      const RowScale s = row_scale(m);
      if (threadIdx.x == 0) xs[t] = s.scale;
      const T* row = source(t);
      if (threadIdx.x * 8 < K) *reinterpret_cast<uint2*>(codes + t * pitch + threadIdx.x * 8) = piece_codes(s, keep[t]);
      for (int k = (512 + threadIdx.x) * 8; k < K; k += 512 * 8) {
        uint32_t v[8];
        row_piece(row, k, Kx, v);
        *reinterpret_cast<uint2*>(codes + t * pitch + k) = piece_codes(s, v);
      }
    }
  }
  __syncthreads();
  const int8_t* const B = codes + min(c, p.N - 1) * pitch;
  i32x4_t acc = {0, 0, 0, 0};
  auto multiply = [&](int s, i32x4_t fa) {
    const int k = 64 * s + 16 * g;
    i32x4_t fb = *reinterpret_cast<const i32x4_t*>(B + min(k, K - 16));
    if (k >= K) fb = i32x4_t{0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa, fb, acc, 0, 0, 0);
  };
  for (int s = wave; s < ns; s += 2 * W) {
    const i32x4_t a0 = a[0], a1 = a[1];
    if (s + 2 * W < ns) a[0] = weight(s + 2 * W);
    if (s + 3 * W < ns) a[1] = weight(s + 3 * W);
    multiply(s, a0);
    if (s + W < ns) multiply(s + W, a1);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || c >= p.N) return;
#pragma unroll
  for (int w = 1; w < W; ++w) acc += part[w][lane];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int v = m0 + 4 * g + q;
    if (v >= p.M) break;
    const float z = float(acc[q]) * xs[c] * p.ws[v];
    if (p.out_bf16) static_cast<uint16_t*>(p.out)[c * p.ldo + v] = f32_to_bf16(z);
    else static_cast<float*>(p.out)[c * p.ldo + v] = z;
  }
}

template <int NT, int MR>
static int launch_skinny(I8Params& p, hipStream_t stream) {
  p.nmb = int32_t((int64_t(p.M) + 16 * MR - 1) / (16 * MR));
  p.nnb = int32_t((p.N + 16 * NT - 1) / (16 * NT));
  const int64_t nblk = (p.nmb < 8 ? p.nmb : rup(p.nmb, 8)) * p.nnb;
  for (int64_t b = 0; b < nblk; b += kMaxBlocks) {
    p.block0 = int32_t(b);
    hipLaunchKernelGGL((i8_skinny_kernel<NT, MR>), dim3(unsigned(std::min(nblk - b, kMaxBlocks))),
                       dim3(512), 0, stream, p);
    FR_LAUNCHED();
  }
  return FASTRL_OK;
}

// Tokens of a tile column, and pieces of each of the last tiles, those past a multiple of 256: the choice
// whose estimated time is least.  A tile takes about 5 us and, per 128 columns of K, the microseconds listed for
// 64 to 256 tokens; 256 run at once.  linear_i8 in bf16, us, columns of 64 / 128 / 192 / 256 tokens:
//   600 x 3584 x 3584 (T x N x K)  25.6 / 28.5 / 33.1 / 41.0     1500 x 1536 x 1536   20.1 / 22.4 / 25.2 / 29.2
//   2309 x 3584 x 3584             69.9 / 54.7 / 43.8 / 48.8     300 x 14336 x 3584   42.8 / 30.6 / 33.6 / 41.1
//   1001 x 10007 x 1001            39.0 / 37.9 / 31.0 / 34.6     4096 x 3584 x 14336  328 / 234 / 255 / 198
//   500 x 30000 x 1536             50.2 / 38.5 / 41.1 / 33.0     2309 x 14336 x 3584  190 / 138 / 118 / 120
// and with the last tiles whole / cut: 256 x 152064 x 3584 173 / 164, 193 x 151936 x 1536 93.2 / 87.5, 700 x
// 100000 x 2048 156 / 154.
struct TilePlan {
  int width, pieces;
  double us;
};
static TilePlan tile_plan(int64_t T, int32_t N, int32_t K) {
  const double per[4] = {0.60, 0.85, 1.10, 1.45}, nk = double((K + 127) / 128);
  const int64_t nmb = (int64_t(N) + kBM - 1) / kBM;
  TilePlan best{256, 1, -1.0};
  for (int w = 4; w >= 1; --w) {
    const int64_t tiles = nmb * ((T + 64 * w - 1) / (64 * w)), last = tiles % 256;
    const int used = int(std::min<int64_t>(w, (T + 63) / 64));
    for (int pieces = 1; pieces <= used && (pieces == 1 || last > 0); pieces *= 2) {
      const int cut = (used + pieces - 1) / pieces;
      const double t = double(tiles / 256) * (5.0 + nk * per[used - 1]) +
                       double((last * pieces + 255) / 256) * (5.0 + nk * per[cut - 1]) * (pieces > 1 ? 1.02 : 1.0);
      if (best.us < 0.0 || t < best.us) best = {64 * w, pieces, t};
    }
  }
  return best;
}

// Channels (in 16s) of a block of the kernel for few tokens and channels, 0: whole tiles.  linear_i8 in bf16,
// us, whole tiles / 1 / 2 / 4 (with ~13 us of the caller's time; quantisation included):
//   N x K        T = 1                       16                      64                     128
//   1536 x 1536   14.7 / 14.5 / 14.0 / 14.6   15.1 / 14.4 / 14.7 / 14.8   15.6 / 14.4 / 14.5 / 15.1   14.9 / 14.3 / 14.4 / 13.9
//   3584 x 3584   21.6 / 14.1 / 14.2 / 14.7   22.6 / 14.6 / 14.2 / 15.2   22.9 / 16.6 / 17.9 / 21.2   23.3 / 23.6 / 18.0 / 21.1
//   3584 x 14336  66.5 / 20.2 / 23.7 / 35.7   67.1 / 22.6 / 28.2 / 40.3   68.0 / 42.0 / 47.8 / 61.1   67.7 / 73.2 / 48.2 / 60.8
//   14336 x 3584  22.5 / 15.4 / 14.8 / 14.5   22.8 / 19.7 / 17.0 / 15.5   23.3 / 39.8 / 27.4 / 22.0
//   30000 x 1536  15.9 / 15.6 / 14.3 / 14.5   16.1 / 18.2 / 15.9 / 15.4   16.2 / 37.2 / 27.0 / 23.0
//   152064 x 3584 109 / 98.6 / 102 / 105      111 / 162 / 138 / 125       119 / 346 / 227 / 189
// and 256 tokens of 3584 x 3584 23.6 / 39.7 / 27.9 / 21.9, of 3584 x 14336 68.5 / 134 / 85.8 / 61.2.
struct SkinnyPlan {
  int rows, tokens;  // of a block, in 16s
};
static SkinnyPlan skinny_plan(int64_t T, int32_t N, int32_t K, double tiles_us) {
  // columns of at most 64 tokens, of equal width
  const int64_t cols = (T + 63) / 64;
  const int nt = int(((T + cols - 1) / cols + 15) / 16);
  if (T <= 4) return {N < 8192 ? 1 : 2, nt};
  if (N < 8192 && T <= 256) return {T <= 64 ? 1 : T <= 128 ? 2 : 4, nt};
  if (N >= 8192) return {N < 65536 && (T <= 16 || (T <= 64 && N < 20000)) ? 4 : 0, nt};
  // more tokens, where whole tiles are few: a compute unit reads about 38 bytes of codes a nanosecond.  Whole
  // tiles / so: 297 x 328 x 3923 (T x N x K) 26.2 / 13.6 us, 600 x 328 x 14336 70.8 / 44.5, 1200 x 64 x 3923 27.3 / 13.7,
  // 4096 x 64 x 14336 95.7 / 62.6
  SkinnyPlan best{0, nt};
  double us = tiles_us;
  for (int r = 1; r <= 4; r *= 2)
    for (int n = 1; n <= 4; ++n) {
      const int64_t nmb = (N + 16 * r - 1) / (16 * r);
      const int64_t blocks = (nmb < 8 ? nmb : rup(nmb, 8)) * ((T + 16 * n - 1) / (16 * n));
      const double t = 3.0 + double((blocks + 255) / 256) * (1.5 + K * 16.0 * (r + n) / 38e3);
      if (t < us && blocks < (int64_t(1) << 30)) {
        best = {r, n};
        us = t;
      }
    }
  return best;
}

template <int MR>
static int launch_skinny_tokens(I8Params& p, int nt, hipStream_t stream) {
  return nt == 1   ? launch_skinny<1, MR>(p, stream)
         : nt == 2 ? launch_skinny<2, MR>(p, stream)
         : nt == 3 ? launch_skinny<3, MR>(p, stream)
                   : launch_skinny<4, MR>(p, stream);
}

double i8_tiles_us(int64_t T, int32_t N, int32_t K) { return tile_plan(T, N, K).us; }

int launch_matmul_i8(const I8Call& a, hipStream_t stream) {
  if (a.T == 0) return FASTRL_OK;
  I8Params p{};
  p.A = a.w; p.lda = a.ldw / 2; p.M = a.N;
  p.B = a.x; p.ldb = a.ldx / 2; p.N = int32_t(a.T);
  p.K = a.K / 2;
  p.xs = a.xs; p.ws = a.ws;
  p.out = a.out; p.ldo = a.ldo; p.out_bf16 = a.out_dtype == FASTRL_BF16;
  p.part = a.part; p.ldpart = a.ldpart; p.mask = a.mask; p.bound = a.bound; p.tau2 = a.inv_tau * 1.4426950408889634f;
  const TilePlan plan = tile_plan(a.T, a.N, a.K);
  if (!a.part) {
    const SkinnyPlan s = skinny_plan(a.T, a.N, a.K, plan.us);
    if (s.rows == 1) return launch_skinny_tokens<1>(p, s.tokens, stream);
    if (s.rows == 2) return launch_skinny_tokens<2>(p, s.tokens, stream);
    if (s.rows == 4) return launch_skinny_tokens<4>(p, s.tokens, stream);
  }
  p.staged = ((reinterpret_cast<uintptr_t>(a.out) | uint64_t(a.ldo) * (p.out_bf16 ? 2 : 4)) & 15) != 0;
  p.width = plan.width;
  p.pieces = plan.pieces;
  p.nmb = int32_t((int64_t(a.N) + kBM - 1) / kBM);
  p.nnb = int32_t((a.T + p.width - 1) / p.width);
  p.group = kGroup;
  const int64_t tiles = int64_t(p.nmb) * p.nnb, last = p.pieces > 1 ? tiles % 256 : 0;
  const int64_t nblk = tiles - last + rup(last, 8) * p.pieces;
  FR_CHECK_ARG(nblk < (int64_t(1) << 31), FASTRL_ERR_UNSUPPORTED, "int8 GEMM: grid too large");
  p.whole = int32_t(tiles - last);
  for (int64_t b = 0; b < nblk; b += kMaxBlocks) {
    p.block0 = int32_t(b);
    hipLaunchKernelGGL(a.part ? i8_gemm_kernel<true> : i8_gemm_kernel<false>,
                       dim3(unsigned(std::min(nblk - b, kMaxBlocks))), dim3(kThreads), 0, stream, p);
    FR_LAUNCHED();
  }
  return FASTRL_OK;
}

static int check_product(const char* fn, const void* x, int64_t ldx, const void* w, int64_t ldw,
                         const void* ws, int64_t T, int32_t N, int32_t K, const void* out,
                         int32_t out_dtype, int64_t ldo) {
  const std::string f(fn);
  FR_CHECK_ARG(out_dtype == FASTRL_F32 || out_dtype == FASTRL_BF16, FASTRL_ERR_DTYPE,
               f + ": out_dtype must be FASTRL_F32 or FASTRL_BF16");
  // (a tile's token numbers go past T by less than 256, in 32 bits)
  FR_CHECK_ARG(T >= 0 && T <= (int64_t(1) << 31) - 1024 && N >= 1 && N < (1 << 30), FASTRL_ERR_SHAPE,
               f + ": need 0 <= T <= 2^31 - 1024 and 1 <= N < 2^30");
  FR_CHECK_ARG(K >= 1 && K < 131072, FASTRL_ERR_SHAPE,
               f + ": need 1 <= K < 131072 (sums of 32 bits)");
  const int64_t Kp = rup(K, 16);
  FR_CHECK_ARG(ldw >= Kp && ldw % 16 == 0 && ldw < (int64_t(1) << 28), FASTRL_ERR_SHAPE,
               f + ": ldw must be a multiple of 16, at least K rounded up to 16, below 2^28");
  FR_CHECK_ARG(ldx >= Kp && ldx % 16 == 0, FASTRL_ERR_SHAPE,
               f + ": ldx must be a multiple of 16, at least K rounded up to 16");
  FR_CHECK_ARG(ldo >= N, FASTRL_ERR_SHAPE, f + ": ldo must be at least N");
  if (T == 0) return FASTRL_OK;
  FR_CHECK_ARG(x && w && ws && out, FASTRL_ERR_NULL_PTR, f + ": x / w / w_scale / out is NULL");
  FR_CHECK_ARG((reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (reinterpret_cast<uintptr_t>(w) & 15u) == 0,
               FASTRL_ERR_VALUE, f + ": codes must be 16-byte aligned");
  return FASTRL_OK;
}

// Calls of few tokens and channels code the rows in the kernel that multiplies them and leave the workspace alone.
// linear_i8 in bf16, us, two launches / one (mostly the caller's time): 1 x 1536 x 1536 (T x N x K) 12.2 / 8.9, 16 x
// 1536 x 1536 12.3 / 10.2, 16 x 3584 x 3584 12.2 / 11.2, 8 x 3584 x 6000 12.2 / 11.8.  Not where one wavefront would have
// more than 7168 columns to code (11 x 300 x 5000 12.4 / 13.3, 5 x 300 x 8192 12.3 / 14.5), or the blocks
// together more than 230M (8 x 8000 x 4500 12.1 / 14.7, 16 x 32000 x 1536 13.6 / 28.5).
static bool one_launch(int64_t T, int32_t N, int32_t K) {
  if (T > 16 || N >= 8192 || K > 32768) return false;
  const int64_t Kp = rup(K, 16);
  return T * Kp <= token_codes(int(T)) && (T <= 4 || (T + 7) / 8 * Kp <= 7168) && N * T * Kp <= 230000000;
}

struct LinearWs {
  int8_t* q;
  float* scale;
};

static size_t carve_linear(Carver& c, LinearWs& w, int64_t T, int32_t K) {
  w.q = c.take<int8_t>(size_t(std::max<int64_t>(T, 1) * rup(K, 16)));
  w.scale = c.take<float>(size_t(std::max<int64_t>(T, 1)));
  return c.size();
}

}  // namespace fastrl

using namespace fastrl;

extern "C" {

int fastrl_quantize_rows(const void* x, int32_t dtype, const int32_t* row_index, int64_t T,
                         int32_t K, int64_t ldx, int8_t* q, int64_t ldq, float* scale,
                         hipStream_t stream) {
  clear_error();
  FR_CHECK_ARG(dtype == FASTRL_F32 || dtype == FASTRL_BF16, FASTRL_ERR_DTYPE,
               "fastrl_quantize_rows: dtype must be FASTRL_F32 or FASTRL_BF16");
  FR_CHECK_ARG(T >= 0 && T < (int64_t(1) << 31) && K >= 1, FASTRL_ERR_SHAPE,
               "fastrl_quantize_rows: need 0 <= T < 2^31 and K >= 1");
  FR_CHECK_ARG(ldx >= K && ldq >= K, FASTRL_ERR_SHAPE,
               "fastrl_quantize_rows: ldx and ldq must be at least K");
  if (T == 0) return FASTRL_OK;
  FR_CHECK_ARG(x && q && scale, FASTRL_ERR_NULL_PTR, "fastrl_quantize_rows: x / q / scale is NULL");
  return launch_quantize(x, dtype, row_index, T, K, ldx, q, ldq, scale, stream);
}

int fastrl_matmul_i8(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                     int64_t ldw, const float* w_scale, int64_t T, int32_t N, int32_t K, void* out,
                     int32_t out_dtype, int64_t ldo, hipStream_t stream) {
  clear_error();
  const int rc = check_product("fastrl_matmul_i8", x, ldx, w, ldw, w_scale, T, N, K, out, out_dtype, ldo);
  if (rc != FASTRL_OK) return rc;
  FR_CHECK_ARG(T == 0 || x_scale, FASTRL_ERR_NULL_PTR, "fastrl_matmul_i8: x_scale is NULL");
  I8Call a{};
  a.x = x; a.ldx = ldx; a.xs = x_scale; a.w = w; a.ldw = ldw; a.ws = w_scale;
  a.T = T; a.N = N; a.K = int32_t(rup(K, 16));
  a.out = out; a.out_dtype = out_dtype; a.ldo = ldo;
  return launch_matmul_i8(a, stream);
}

size_t fastrl_linear_i8_workspace_size(int64_t T, int32_t N, int32_t K) {
  if (T < 0 || N < 1 || K < 1 || (T <= 4 && one_launch(T, N, K))) return 0;
  Carver c(nullptr);
  LinearWs w;
  return carve_linear(c, w, T, K);
}

int fastrl_linear_i8(const void* x, int32_t dtype, const int32_t* row_index, int64_t ldx,
                     const int8_t* w, int64_t ldw, const float* w_scale, int64_t T, int32_t N,
                     int32_t K, void* out, int32_t out_dtype, int64_t ldo, void* ws,
                     size_t ws_bytes, hipStream_t stream) {
  clear_error();
  FR_CHECK_ARG(dtype == FASTRL_F32 || dtype == FASTRL_BF16, FASTRL_ERR_DTYPE,
               "fastrl_linear_i8: dtype must be FASTRL_F32 or FASTRL_BF16");
  // (the codes lie in the workspace, which is checked below)
  const int rc = check_product("fastrl_linear_i8", x ? w : nullptr, rup(std::max(K, 1), 16), w, ldw,
                               w_scale, T, N, K, out, out_dtype, ldo);
  if (rc != FASTRL_OK) return rc;
  FR_CHECK_ARG(ldx >= K, FASTRL_ERR_SHAPE, "fastrl_linear_i8: ldx must be at least K");
  if (T == 0) return FASTRL_OK;
  const size_t need = fastrl_linear_i8_workspace_size(T, N, K);
  FR_CHECK_ARG(need == 0 || (ws && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0 && ws_bytes >= need),
               FASTRL_ERR_WORKSPACE,
               "fastrl_linear_i8: workspace missing, misaligned or smaller than " + std::to_string(need) +
                   " bytes");
  const int64_t Kp = rup(K, 16);
  if (one_launch(T, N, K)) {
    I8Params p{};
    p.A = w; p.lda = ldw / 2; p.M = N; p.N = int32_t(T); p.K = int32_t(Kp / 2); p.ws = w_scale;
    p.out = out; p.ldo = ldo; p.out_bf16 = out_dtype == FASTRL_BF16;
    const dim3 grid(unsigned((N + 15) / 16));
    auto launch = [&](auto rows) {
      using T_ = std::remove_const_t<std::remove_pointer_t<decltype(rows)>>;
      hipLaunchKernelGGL((T <= 4 ? i8_token_kernel<T_, 4> : i8_token_kernel<T_, 16>), grid, dim3(512), 0, stream, p,
                         rows, row_index, ldx, K);
    };
    if (dtype == FASTRL_BF16) launch(static_cast<const uint16_t*>(x));
    else launch(static_cast<const float*>(x));
    FR_LAUNCHED();
    return FASTRL_OK;
  }
  Carver c(ws);
  LinearWs l;
  carve_linear(c, l, T, K);
  const int rq = launch_quantize(x, dtype, row_index, T, K, ldx, l.q, Kp, l.scale, stream);
  if (rq != FASTRL_OK) return rq;
  I8Call a{};
  a.x = l.q; a.ldx = Kp; a.xs = l.scale; a.w = w; a.ldw = ldw; a.ws = w_scale;
  a.T = T; a.N = N; a.K = int32_t(Kp);
  a.out = out; a.out_dtype = out_dtype; a.ldo = ldo;
  return launch_matmul_i8(a, stream);
}

}  // extern "C"
