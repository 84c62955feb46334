// Writing a cache in 8 or 4 bits, and reading it back (formats in quant.hpp).
//
// Both are byte work bound by memory: 16 lanes take a row, 16 bytes of bf16 each.  The maximum of a block of 32
// elements (4 lanes) is taken on the bf16 bit patterns with the sign cleared, whose order as integers is that of
// the magnitudes, with infinities and NaNs above every finite value; its exponent field gives the scale byte and
// its mantissa the one case in which the next exponent is taken.  Codes come from the conversion instructions
// (nearest, ties to even) of x * 2^-e, which is exact.  A 16K x 8 prompt is written in 4 bits in 120 us (5.1 TB/s read
// and written, a copy's rate) and read back in 96 us (6.6 TB/s, the codes partly in the caches) to 115.

#include "bd_common.hpp"
#include "bd_kernels.hpp"
#include "quant.hpp"

namespace bd {
namespace {

constexpr int kThreads = 256;
constexpr int kRowLanes = 16;                  // lanes of a row, 8 elements each
constexpr int kRowsAtOnce = kThreads / kRowLanes;
constexpr int kFusedRows = 16;                 // appends of up to this many rows advance the lengths in the same launch
// 6 rows of 32 heads, 64 sequences, 8 bits: 9.7 us with 512 threads, 8.6 with 1024; one row of 8 heads 3.1 us with both.
// The rows' arithmetic on one CU a sequence bounds the larger: loads issued 2, 3 or 6 rows ahead change nothing.
constexpr int kFusedThreads = 1024;
// Rows of one head that a workgroup of the longer calls takes.  Written, 32 / 64 / 128 rows: 16K x 8 prompts written
// and read back in 243 / 243 / 253 us; read back, 16 / 32 / 64 / 128: 16K x 8 in 126 / 115 / 123 / 131 us, in 16-row
// pages 168 / 147 / 151 / 151.
constexpr int kWriteRows = 64, kReadRows = 32;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The new rows are read once, the rows read back go to a buffer larger than the caches: non-temporal.
__device__ inline u32x4 load16_nt(const uint16_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
__device__ inline void store16_nt(uint16_t* p, const u32x4& v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }

template <int CTRL>
__device__ inline uint32_t max_dpp(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
  return x > y ? x : y;
}

// Codes of this lane's 8 elements (4 or 8 bytes, in c[0] and c[1]) and the scale byte of its block (the 4 lanes of
// a quad).  Every lane of the quad takes part.
template <int BITS>
__device__ inline int quantise8(const u32x4& w, uint32_t (&c)[2]) {
  using F = QFormat<BITS>;
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  uint32_t a = m[0] > m[1] ? m[0] : m[1];
  a = max_dpp<0xB1>(a);                        // quad_perm [1,0,3,2]
  a = max_dpp<0x4E>(a);                        // quad_perm [2,3,0,1]
  const int E = (int)(a >> 7);                 // biased exponent
  c[0] = c[1] = 0u;
  if (E == 255) return kScaleNan;
  int byte = E - F::kEmax + ((int)(a & 127u) > F::kTopMant ? 1 : 0);
  byte = byte < F::kByteMin ? F::kByteMin : (byte > F::kByteMax ? F::kByteMax : byte);
  const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(w[i]) * inv;
    x[2 * i + 1] = bf16_hi(w[i]) * inv;
  }
  if constexpr (BITS == 4) {
    // saturates at 6
    c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[0], x[0], x[1], 1.f, 0);
    c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[0], x[2], x[3], 1.f, 1);
    c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[0], x[4], x[5], 1.f, 2);
    c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[0], x[6], x[7], 1.f, 3);
  } else {
    // does not saturate: only at the clamped exponent does an element exceed 464
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int y = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
      c[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], y, true);
    }
  }
  return byte;
}

// The scale bytes of a row's four quads in one word, in every lane of the 16.
template <int CTRL>
__device__ inline uint32_t or_dpp(uint32_t x) { return x | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false); }
__device__ inline uint32_t row_scales(int byte, int j) {
  const uint32_t x = (uint32_t)byte << (8 * (j >> 2));
  return or_dpp<0x128>(or_dpp<0x124>(x));      // rows of 16 lanes turned by 4, then by 8
}

// This lane's part (elements 8*j .. 8*j+7) of row `row` from 16 bytes of bf16.  All 16 lanes of the row take part.
template <int BITS>
__device__ inline void write_row(uint8_t* codes, uint8_t* scales, int64_t row, int j, const u32x4& w) {
  uint32_t c[2];
  const uint32_t sc = row_scales(quantise8<BITS>(w, c), j);
  uint8_t* dst = codes + row * QFormat<BITS>::kRow + BITS * j;
  if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(dst) = c[0];
  else *reinterpret_cast<uint64_t*>(dst) = (uint64_t)c[0] | ((uint64_t)c[1] << 32);
  if (j == 0) *reinterpret_cast<uint32_t*>(scales + row * kBlocks) = sc;
}

// Rows that sequence s gets.
__device__ inline int new_rows(const QAppendParams& p, int s) {
  if (!p.counts) return p.n;
  const int c = p.counts[s];
  return c < 0 ? 0 : (c > p.n ? p.n : c);
}

__device__ inline int list_count(const QAppendParams& p, int s) {
  const int m = p.nsel[s];
  return m < 0 ? 0 : (m > p.ld_idx ? p.ld_idx : m);
}

// Advance sequence s's length (and sparse count) by the rows written.
__device__ inline void advance(const QAppendParams& p, int s, int L, int n) {
  const int cap = p.kv.max_seq_len;
  const int w = n < cap - L ? n : cap - L;
  const_cast<int32_t*>(p.kv.seq_lens)[s] = L + w;
  if (p.idx) {
    const int m = list_count(p, s);
    p.nsel[s] = m + (w < p.ld_idx - m ? w : p.ld_idx - m);
  }
}

// Block s: every new row of sequence s (n <= kFusedRows), then its length.  All reads of the old length and
// count happen before the barrier; thread 0 writes the new ones after it.
template <int BITS>
__global__ __launch_bounds__(kFusedThreads) void append_q_fused_kernel(QAppendParams p) {
  const int s = blockIdx.x;
  const int cap = p.kv.max_seq_len, Hkv = p.kv.num_kv_heads;
  const int L = seq_len(p.kv, s), n = new_rows(p, s);
  const int m = p.idx ? list_count(p, s) : 0;
  const int j = threadIdx.x % kRowLanes;
  __shared__ int64_t rows[kFusedRows];                      // of head 0; -1: past the capacity or the pool, dropped
  if ((int)threadIdx.x < n) rows[threadIdx.x] = L + (int)threadIdx.x < cap ? row_of(p.kv, s, L + (int)threadIdx.x) : -1;
  __syncthreads();
  // work item: (new row i, head and K or V r), 16 lanes each, kItems at a time; the next one's i and r by addition
  constexpr int kItems = kFusedThreads / kRowLanes;
  const int per = 2 * Hkv, di = kItems / per, dr = kItems - di * per;
  const int first = threadIdx.x / kRowLanes;
  int i = first / per, r = first - i * per;
  while (i < n) {                                           // whole rows leave the loop together
    const int g = r >> 1;
    const bool is_v = r & 1;
    if (rows[i] >= 0) {
      const u32x4 src = load16((is_v ? p.v_new : p.k_new) + (((int64_t)s * p.n + i) * Hkv + g) * kD + 8 * j);
      write_row<BITS>(is_v ? p.kv.v : p.kv.k, is_v ? p.kv.v_scale : p.kv.k_scale, rows[i] + (int64_t)g * p.kv.stride_head, j,
                      src);
    }
    i += di;
    r += dr;
    if (r >= per) {
      r -= per;
      ++i;
    }
  }
  if (p.idx)
    for (int w = threadIdx.x; w < n * Hkv; w += kFusedThreads) {
      const int i = w / Hkv, g = w - i * Hkv;
      if (L + i < cap && m + i < p.ld_idx) p.idx[((int64_t)s * Hkv + g) * p.ld_idx + m + i] = L + i;
    }
  __syncthreads();
  if (threadIdx.x == 0) advance(p, s, L, n);
}

// A workgroup takes kWriteRows new rows of one (sequence, head), K and V.
template <int BITS>
__global__ __launch_bounds__(kThreads) void append_q_rows_kernel(QAppendParams p, int64_t groups, int per_head) {
  const int cap = p.kv.max_seq_len, Hkv = p.kv.num_kv_heads;
  const int j = threadIdx.x % kRowLanes;
  for (int64_t b = blockIdx.x; b < groups; b += gridDim.x) {
    const int64_t pair = b / per_head;
    const int i0 = (int)(b - pair * per_head) * kWriteRows;
    const int s = (int)(pair / Hkv), g = (int)(pair - (int64_t)s * Hkv);
    const int L = seq_len(p.kv, s), n = new_rows(p, s);
    // every row's loads are issued before the first is used
    constexpr int kPer = kWriteRows / kRowsAtOnce;
    u32x4 kw[kPer], vw[kPer];
    int64_t row[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = i0 + threadIdx.x / kRowLanes + u * kRowsAtOnce;
      const int64_t t = (int64_t)L + i;
      row[u] = i < n && t < cap ? row_of(p.kv, s, (int)t) : -1;
      if (row[u] < 0) continue;
      const int64_t src = (((int64_t)s * p.n + i) * Hkv + g) * kD + 8 * j;
      kw[u] = load16_nt(p.k_new + src);
      vw[u] = load16_nt(p.v_new + src);
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      if (row[u] < 0) continue;                            // past the new rows, the capacity or the pool
      const int64_t at = row[u] + (int64_t)g * p.kv.stride_head;
      write_row<BITS>(p.kv.k, p.kv.k_scale, at, j, kw[u]);
      write_row<BITS>(p.kv.v, p.kv.v_scale, at, j, vw[u]);
    }
    if (p.idx) {
      const int m = list_count(p, s);
      for (int i = i0 + threadIdx.x; i < i0 + kWriteRows; i += kThreads)
        if (i < n && L + i < cap && i < p.ld_idx - m) p.idx[((int64_t)s * Hkv + g) * p.ld_idx + m + i] = L + i;
    }
  }
}

// Thread s: advance the length (and the sparse count) by what append_q_rows_kernel wrote.
__global__ __launch_bounds__(kThreads) void append_q_advance_kernel(QAppendParams p) {
  const int s = blockIdx.x * kThreads + threadIdx.x;
  if (s < p.kv.num_seqs) advance(p, s, seq_len(p.kv, s), new_rows(p, s));
}

// 16 bytes of bf16 from this lane's 8 codes (c) and its block's scale byte.
template <int BITS>
__device__ inline u32x4 dequantise8(const uint32_t (&c)[2], int byte) {
  const float sc = __uint_as_float((uint32_t)byte << 23);   // 255: not a number, as every value of the block
  u32x4 w;
  if constexpr (BITS == 4) {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], sc, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], sc, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], sc, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], sc, 3));
  } else {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], sc, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], sc, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], sc, 0));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], sc, 1));
  }
  return w;
}

// This lane's codes and its block's scale byte of a row.
template <int BITS>
struct Part { uint32_t c[2]; int byte; };
template <int BITS>
__device__ inline Part<BITS> read_part(const uint8_t* codes, const uint8_t* scales, int64_t row, int j) {
  const uint8_t* src = codes + row * QFormat<BITS>::kRow + BITS * j;
  Part<BITS> r{{0u, 0u}, scales[row * kBlocks + (j >> 2)]};
  if constexpr (BITS == 4) {
    r.c[0] = *reinterpret_cast<const uint32_t*>(src);
  } else {
    const uint64_t x = *reinterpret_cast<const uint64_t*>(src);
    r.c[0] = (uint32_t)x;
    r.c[1] = (uint32_t)(x >> 32);
  }
  return r;
}

// A workgroup takes kReadRows output rows of one (sequence, head); rows that the cache does not hold become zero.
template <int BITS>
__global__ __launch_bounds__(kThreads) void read_q_kernel(QReadParams p, int64_t groups, int per_head) {
  const int Hkv = p.kv.num_kv_heads;
  const int j = threadIdx.x % kRowLanes;
  for (int64_t b = blockIdx.x; b < groups; b += gridDim.x) {
    const int64_t pair = b / per_head;
    const int i0 = (int)(b - pair * per_head) * kReadRows;
    const int s = (int)(pair / Hkv), g = (int)(pair - (int64_t)s * Hkv);
    const int L = seq_len(p.kv, s);
    const int f = p.first ? p.first[s] : 0;
    // every row's loads are issued before the first is used
    constexpr int kPer = kReadRows / kRowsAtOnce;
    Part<BITS> kp[kPer], vp[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = i0 + threadIdx.x / kRowLanes + u * kRowsAtOnce;
      const int64_t t = (int64_t)f + i;
      int64_t row = i < p.n && t >= 0 && t < L ? row_of(p.kv, s, (int)t) : -1;
      kp[u] = vp[u] = Part<BITS>{{0u, 0u}, QFormat<BITS>::kByteMin};       // zeros
      if (row < 0) continue;
      row += (int64_t)g * p.kv.stride_head;
      if (p.k_out) kp[u] = read_part<BITS>(p.kv.k, p.kv.k_scale, row, j);
      if (p.v_out) vp[u] = read_part<BITS>(p.kv.v, p.kv.v_scale, row, j);
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = i0 + threadIdx.x / kRowLanes + u * kRowsAtOnce;
      if (i >= p.n) break;
      const int64_t dst = (int64_t)s * p.stride_seq + (int64_t)g * p.stride_head + (int64_t)i * p.stride_tok + 8 * j;
      if (p.k_out) store16_nt(p.k_out + dst, dequantise8<BITS>(kp[u].c, kp[u].byte));
      if (p.v_out) store16_nt(p.v_out + dst, dequantise8<BITS>(vp[u].c, vp[u].byte));
    }
  }
}

constexpr int64_t kMaxGrid = 1 << 22;          // larger calls loop

}  // namespace

hipError_t launch_append_q(const QAppendParams& p, int bits, hipStream_t stream) {
  const unsigned S = (unsigned)p.kv.num_seqs;
  if (p.n <= kFusedRows) {
    if (bits == 4) hipLaunchKernelGGL((append_q_fused_kernel<4>), dim3(S), dim3(kFusedThreads), 0, stream, p);
    else hipLaunchKernelGGL((append_q_fused_kernel<8>), dim3(S), dim3(kFusedThreads), 0, stream, p);
    return hipGetLastError();
  }
  const int per_head = (p.n + kWriteRows - 1) / kWriteRows;
  const int64_t groups = (int64_t)S * p.kv.num_kv_heads * per_head;
  const dim3 grid((unsigned)(groups < kMaxGrid ? groups : kMaxGrid));
  if (bits == 4) hipLaunchKernelGGL((append_q_rows_kernel<4>), grid, dim3(kThreads), 0, stream, p, groups, per_head);
  else hipLaunchKernelGGL((append_q_rows_kernel<8>), grid, dim3(kThreads), 0, stream, p, groups, per_head);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(append_q_advance_kernel, dim3((S + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_read_q(const QReadParams& p, int bits, hipStream_t stream) {
  const int per_head = (p.n + kReadRows - 1) / kReadRows;
  const int64_t groups = (int64_t)p.kv.num_seqs * p.kv.num_kv_heads * per_head;
  const dim3 grid((unsigned)(groups < kMaxGrid ? groups : kMaxGrid));
  if (bits == 4) hipLaunchKernelGGL((read_q_kernel<4>), grid, dim3(kThreads), 0, stream, p, groups, per_head);
  else hipLaunchKernelGGL((read_q_kernel<8>), grid, dim3(kThreads), 0, stream, p, groups, per_head);
  return hipGetLastError();
}

}  // namespace bd
