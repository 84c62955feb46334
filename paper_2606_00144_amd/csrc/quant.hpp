// A KV cache held in 8 or 4 bits: the formats and the parameter blocks of its kernels.
//
// A row of 128 elements is 128 e4m3 codes (8 bits) or 64 bytes of e2m1 codes (4 bits, the even element in the low
// half), with one E8M0 byte per block of 32 elements: value = code * 2^(byte - 127) (the microscaling formats MXFP8
// and MXFP4).  Powers of two as scales make x * 2^-e exact, so a code is defined to the bit by its element and its
// block's maximum, and every value is exact in bf16: 4 significand bits at most, in the normal range.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "bd_common.hpp"

namespace bd {

constexpr int kBlocks = kD / 32;               // scale bytes per row

template <int BITS>
struct QFormat {
  static_assert(BITS == 8 || BITS == 4, "e4m3 or e2m1");
  static constexpr int kRow = kD * BITS / 8;                 // bytes of a row of codes
  static constexpr int kEmax = BITS == 8 ? 8 : 2;            // exponent of the largest binade
  // a block whose maximum lies above this mantissa (7 bits) takes the next exponent: 464 = 1.8125 * 2^8 and
  // 7 = 1.75 * 2^2 lie half a step above the largest values 448 and 6
  static constexpr int kTopMant = BITS == 8 ? 104 : 96;
  static constexpr int kByteMin = 16;                        // 2^-111: the smallest value, 2^-9 of it, is a normal bf16
  static constexpr int kByteMax = 254 - kEmax;               // the largest value stays finite
};
constexpr int kScaleNan = 255;                               // scale byte of a block that held a NaN or an infinity

// Device copy of bd_qkv_desc.  Rows of codes and of scales share one numbering: row r has its codes at
// r * QFormat::kRow and its scales at 4 * r; strides count rows.
struct QView {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  const int32_t* seq_lens;
  const int32_t* page_table;
  int64_t stride_seq, stride_head, stride_tok, stride_page;
  int32_t num_seqs, num_kv_heads, max_seq_len;
  int32_t page_size, max_pages_per_seq, num_pages;
};

__device__ inline int seq_len(const QView& kv, int s) {
  const int L = kv.seq_lens[s];
  return L < 0 ? 0 : (L > kv.max_seq_len ? kv.max_seq_len : L);
}

// Row number of position t of head 0 of sequence s, or -1 when its page is outside the pool.
__device__ inline int64_t row_of(const QView& kv, int s, int t) {
  if (kv.page_table) {
    const int pg = kv.page_table[(int64_t)s * kv.max_pages_per_seq + t / kv.page_size];
    return (unsigned)pg < (unsigned)kv.num_pages ? (int64_t)pg * kv.stride_page + (int64_t)(t % kv.page_size) * kv.stride_tok
                                                 : -1;
  }
  return (int64_t)s * kv.stride_seq + (int64_t)t * kv.stride_tok;
}

// ---- writing and reading back ------------------------------------------------
struct QAppendParams {
  QView kv;                 // the cache written (seq_lens advanced in place)
  const uint16_t* k_new;    // [S][n][Hkv][D]
  const uint16_t* v_new;
  int32_t n;
  const int32_t* counts;    // nullable [S]: rows of each sequence that exist (at most n)
  int32_t* idx;             // nullable [S][Hkv][ld_idx]
  int32_t* nsel;
  int32_t ld_idx;
};
hipError_t launch_append_q(const QAppendParams& p, int bits, hipStream_t stream);

struct QReadParams {
  QView kv;
  const int32_t* first;     // nullable [S]
  int32_t n;
  uint16_t* k_out;          // either may be NULL
  uint16_t* v_out;
  int64_t stride_seq, stride_head, stride_tok;   // of the outputs, elements
};
hipError_t launch_read_q(const QReadParams& p, int bits, hipStream_t stream);

// ---- attention ------------------------------------------------------------------
// How a workgroup finds the rows of its keys: computed (contiguous range), through a table of its pages (pages of
// whole 16-row sub-tiles), or through a table of its rows (gathered entries, other page sizes).
enum QRows { kQContiguous = 0, kQPages = 1, kQTable = 2 };

struct QAttnParams {
  QView kv;
  const uint16_t* q;        // [S][nq][Hq][D]
  uint16_t* out;            // [S][nq][Hq][D]
  float* lse;               // nullable [S][nq][Hq]
  const int32_t* idx;       // gathered: [S][Hkv][ld_idx] (NULL: the cache's first L_s rows)
  const int32_t* nsel;      // gathered: [S]
  int32_t ld_idx;
  int32_t S, Hkv, Hq, G;
  int32_t nq;               // query rows per head
  int32_t R;                // rows per (s, g): nq * G
  int32_t n_rb;             // row blocks
  int32_t nW;               // shares of the key stream
  float scale_log2;         // softmax scale * log2(e)
  float* part;              // partial records: two per workgroup
  uint32_t part_bytes;
  uint32_t* counters;
};

struct QAttnPlan {
  int nt, n_rb, R, nW;
  QRows rows;
  int64_t nblk;             // workgroups, -1: too many
  size_t counter_bytes, record_bytes, ws_bytes;
};

// `entries`: the list's width (gathered) or the largest length.
QAttnPlan plan_qattn(int S, int Hkv, int Hq, int nq, int64_t entries, bool gather, bool paged, int page_size);
hipError_t launch_qattn(const QAttnParams& p, const QAttnPlan& pl, int bits, hipStream_t stream);

}  // namespace bd
