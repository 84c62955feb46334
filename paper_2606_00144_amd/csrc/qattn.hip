// Attention of a small block of query rows over a cache held in 8 or 4 bits (formats in quant.hpp): the verifier's
// gamma+1 positions over the whole cache, and the drafter's position over selected entries.
//
// Mathematics.  For a KV head's R = nq * G query rows, scores S^T[key][row] = K . Q^T and outputs O^T[d][row] +=
// V^T . P^T run on v_mfma_f32_16x16x32_bf16, with an online softmax whose reference maximum is raised lazily (by
// more than kSlack).  Lane l holds row l%16 of the products' columns and the 8 keys 16h + 4*(l/16) + i of a 32-key
// tile, so the weights of its scores are the second product's operand as they are.  Codes become bf16 on the way to
// the products, exactly (values have at most 4 significand bits and a power-of-two scale; the conversion
// instructions take the scale's exponent and run at full rate).  The scaled 8- and 4-bit MFMA would take K's codes
// as they are, with Q split in two e4m3 terms, at the same matrix time, but its sums were off by up to 1.5e-4 of
// the products' magnitudes (about 2^-13) on random codes, which a log-sum-exp in fp32 shows; it is not used.
//
// Rounding: weights enter the second product in bf16, and the normaliser sums exactly the rounded weights; the
// scores, the statistics, the outputs and the partial records are fp32.
//
// What bounds it.  The codes: 68 (4 bits) or 132 bytes a key for K and V each against 512 operations and a query
// row.  A wave streams its tiles through a ring of two in LDS of its own with direct loads, while the 8 waves of a CU
// (two workgroups) convert and multiply: 32 heads x 64 sequences of 4 bits in pages run at 6.0 to 6.25 TB/s (a bare
// read reaches 6.05), 16K x 8 with 24 rows at 5.7 in the loop (4 bits: MFMA 17%, VALU 40% busy) and 36 us in all,
// 8 bits at 5.3 and 52 us.  A prologue takes 2 us, the four waves' merge 1.3, a level of records 2.5.  Rows beyond 32
// (48 in long streams) are another block, which reads and converts again.  The query rows lie in LDS too: of rows in registers the
// compiler waited for all loads at their first use, in every turn of the loop.  Nothing is kept in scratch memory: a
// wave's first access to it takes 2 to 15 us.
//
// Work decomposition.  All (sequence, KV head) units' tiles form one stream, which is cut into nW equal shares from
// the lengths on the device; workgroup (share, row block) takes the units that its share meets, one after the
// other (short units whole; and each unit gets shares of its own where that is nearly as even).  A share's time
// depends on the lengths as they are, not on the capacity or on the longest sequence.  A
// unit that lies in one share is finished there; the pieces of one cut by share borders leave partial records,
// merged in order by the last workgroup to arrive (units of more than kGroup pieces in two levels), so results do
// not depend on the order of arrival.

#include "bd_common.hpp"
#include "bd_kernels.hpp"
#include "attn_tile.hpp"
#include "quant.hpp"

namespace bd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kTile = 32;                      // keys per wave step
constexpr int kGroup = 8;                      // records merged by one workgroup at a time
// Shares are at least kMinSpan tiles long, a unit counts as that many even if it has fewer (its prologue and merge take
// the time of about that many), and a unit of fewer than kWhole tiles is not cut: the share that has the larger part
// of it takes it.  Shares of at least 4 / 8 / 16 / 24 tiles: 8 heads of one 8K sequence 14.9 / 13.5 / 15.4 / 20.6 us,
// one 4K decode of 2 heads 10.1 / 9.2 / 11.5 / 11.5.
constexpr int kMinSpan = 8, kWhole = 16, kLonger = 6;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;                  // lazy-rescale headroom, log2 units
constexpr uint32_t kAbsent = 0xFFFFFFFFu;

// A tile in LDS: K's codes, V's codes, then the 32 scale words of K and of V.
template <int BITS>
struct Tile {
  static constexpr int kRow = QFormat<BITS>::kRow;
  static constexpr int kParts = kRow / 64;               // 1 KiB loads per 16 rows of K or V
  static constexpr int kLoads = 4 * kParts + 1;          // loads of a tile
  static constexpr int kV = kTile * kRow, kS = 2 * kV, kBytes = kS + 2 * kTile * kBlocks;
  // Load (h, e) of K brings rows of sub-tile h whole: lane l's 16 bytes land at 1024*(kParts*h + e) + 16*l, in row
  // slot l/4 (4 bits; 8e + l/8 with 8).  K's row r takes slot r, its chunk c position c ^ swizzle, so that 16 lanes
  // reading the same chunk of 16 rows meet no bank twice.  V's row 4a + b takes slot 4b + a, so that the 64 lanes
  // reading row 4*(l/16) + b read 64 consecutive words.
  __device__ static int k_row(int l, int e) { return BITS == 4 ? l >> 2 : 8 * e + (l >> 3); }
  __device__ static int k_chunk(int l, int e) { return BITS == 4 ? (l & 3) ^ ((l >> 4) & 3) : (l & 7) ^ (4 * e + (l >> 4)); }
  __device__ static int v_row(int l, int e) {
    return BITS == 4 ? 4 * ((l >> 2) & 3) + (l >> 4) : 4 * ((l >> 3) & 3) + 2 * e + (l >> 5);
  }
  __device__ static int v_chunk(int l) { return l & (kRow / 16 - 1); }
  // byte of chunk c of K's row r (0 <= r < 32)
  __device__ static int k_at(int r, int c) {
    return kRow * r + 16 * (c ^ (BITS == 4 ? (r >> 2) & 3 : (r >> 1) & 7));
  }
};

// Workgroups that share a CU (and with them the waves of a SIMD), and the entries of a workgroup's table.
constexpr int kRing = 2;                       // tile slots of a wave
constexpr int kMaxBlocks = 512;                // workgroups of a launch
template <int BITS, int NT, int ROWS>
struct Config {
  static constexpr int kPerCu = BITS == 8 || NT > 1 ? 2 : 3;
  static constexpr int kPart = NT == 3 ? 1 : NT;       // row tiles whose states meet in LDS at a time
  static constexpr int kTab = ROWS == kQContiguous ? 4 : ROWS == kQPages ? (NT == 3 ? 256 : 448) : BITS == 8 || NT > 1 ? 1024 : 2048;
};

template <int BITS, int NT, int ROWS>
struct Smem {
  alignas(16) uint32_t tab[Config<BITS, NT, ROWS>::kTab];
  union {
    alignas(64) uint8_t ring[kWaves][kRing][Tile<BITS>::kBytes];
    float o[kWaves][16 * Config<BITS, NT, ROWS>::kPart][kD + 4];   // the waves' states, when they merge
  } u;
  union {
    alignas(64) uint8_t q[16 * NT][kD * 2];    // query rows, chunk c (16 bytes) of row r at position c ^ k_swizzle(r % 16)
    struct { float m[kWaves][16 * NT], l[kWaves][16 * NT], lx[kWaves][16 * NT]; } stat;
  } r;
  int32_t rowpos[16 * NT];    // position of each query row (INT_MAX: sees every key)
  int32_t nan_from[kBlocks];  // first position whose V holds not-a-numbers in block b (INT_MAX: none)
  int32_t last;
  int32_t first_hole;         // first tile of the table with an absent key
};

template <int NT>
struct RowState {
  f32x4 o[NT][8];     // O^T[d-tile][row tile]: register i of d-tile dt holds d = 32*(l/16) + 8*i + dt
  float m[NT];        // reference maximum (log2 domain)
  float l[NT];        // this lane's sum of the rounded weights
  float lx[NT];       // and of the unrounded ones (log-sum-exp only)
};

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ inline uint32_t as_word(const bf16x2& v) { return __builtin_bit_cast(uint32_t, v); }

// 8 values of a row as bf16 from their codes (c: one word with 4 bits, two with 8) and the scale's exponent bits.
template <int BITS>
__device__ inline u32x4 to_bf16(uint32_t c0, uint32_t c1, uint32_t scale_bits) {
  const float sc = __uint_as_float(scale_bits);
  if constexpr (BITS == 4)
    return u32x4{as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, sc, 0)), as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, sc, 1)),
                 as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, sc, 2)), as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, sc, 3))};
  else
    return u32x4{as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, sc, 0)), as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, sc, 1)),
                 as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, sc, 0)), as_word(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, sc, 1))};
}

// A tile's codes and scales in registers.
template <int BITS>
struct TileRegs {
  u32x4 k[2][Tile<BITS>::kParts];   // [sub-tile]: 32 elements of key l%16, block l/16
  uint32_t ks[2];                   // their scale's exponent bits
  uint32_t v[8][Tile<BITS>::kParts];// key slot i: 8 elements, d = 8*(l%16) ..
  uint32_t vs[8];                   // their scale byte at the exponent's place (other bits: neighbours')
};

template <int BITS>
__device__ inline void read_tile(TileRegs<BITS>& T, const uint8_t* t, int lane) {
  using L = Tile<BITS>;
  const int lg = lane >> 4, lr = lane & 15;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < L::kParts; ++e)
      T.k[h][e] = *reinterpret_cast<const u32x4*>(t + L::k_at(16 * h + lr, L::kParts * lg + e));
    T.ks[h] = (uint32_t)t[L::kS + 64 * h + 4 * lr + lg] << 23;
    const u32x4 s = *reinterpret_cast<const u32x4*>(t + L::kS + 128 + 64 * h + 16 * lg);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // the byte of block lr/4 to bits 23..30; the conversions look at no other bit
      T.vs[4 * h + i] = __builtin_rotateleft32(s[i], (23u - 8u * (uint32_t)(lr >> 2)) & 31u);
#pragma unroll
      for (int e = 0; e < L::kParts; ++e)
        T.v[4 * h + i][e] = *reinterpret_cast<const uint32_t*>(t + L::kV + 1024 * L::kParts * h + 256 * L::kParts * i +
                                                               4 * L::kParts * lane + 4 * e);
    }
  }
}

// One tile of one wave.  DIRTY: some key of the tile is absent or hidden from some row; key slot i of this lane is
// absent unless bit i of `there`, and lies at position pos0 + 16*(i/4) + i%4.
template <int BITS, int NT, bool DIRTY, bool LSE>
__device__ inline void tile_step(RowState<NT>& st, TileRegs<BITS>& T, const uint8_t (*q)[kD * 2], float scale_log2,
                                 uint32_t there, int pos0, int lane, const int32_t* rowpos, int32_t* nan_from) {
  if constexpr (DIRTY) {
    // What lies in absent rows (stale memory) must not reach the product: 0 * NaN.  Nor may a block that is not a
    // number reach rows that do not see its key: it is taken out, and the first position of such blocks is kept,
    // from which on the rows' outputs become not a number when the waves merge.
    int first = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool present = (there >> i) & 1u, bad = (T.vs[i] & 0x7F800000u) == 0x7F800000u;
      if (present && bad && pos0 + 16 * (i >> 2) + (i & 3) < first) first = pos0 + 16 * (i >> 2) + (i & 3);
#pragma unroll
      for (int e = 0; e < Tile<BITS>::kParts; ++e) T.v[i][e] = present && !bad ? T.v[i][e] : 0u;
      T.vs[i] = present && !bad ? T.vs[i] : 0x3F800000u;
    }
    if (first != 0x7FFFFFFF) atomicMin(&nan_from[(lane & 15) >> 2], first);
  }
  const int lg = lane >> 4, lr = lane & 15;
  f32x4 sc[2][NT];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sc[h][nt] = zero4();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bf16x8 kop[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (BITS == 4) kop[h] = as_bf16x8(to_bf16<4>(T.k[h][0][j], 0u, T.ks[h]));
      else kop[h] = as_bf16x8(to_bf16<8>(T.k[h][j >> 1][2 * (j & 1)], T.k[h][j >> 1][2 * (j & 1) + 1], T.ks[h]));
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const bf16x8 qop = *reinterpret_cast<const bf16x8*>(&q[16 * nt + lr][16 * ((4 * lg + j) ^ k_swizzle(lr))]);
#pragma unroll
      for (int h = 0; h < 2; ++h) sc[h][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[h], qop, sc[h][nt], 0, 0, 0);
    }
  }
  if constexpr (DIRTY) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int last = rowpos[16 * nt + lr];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(((there >> i) & 1u) && pos0 + 16 * (i >> 2) + (i & 3) <= last)) sc[i >> 2][nt][i & 3] = -INFINITY;
    }
  }

  // The reference maximum is raised when a score exceeds it by more than kSlack: the lanes look at their own scores,
  // and only then at each other's.
  float mx[NT];
  bool raise = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float x = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) x = fmaxf(x, sc[i >> 2][nt][i & 3]);
    mx[nt] = x * scale_log2;                          // scale > 0: the max commutes with it
    raise |= mx[nt] > st.m[nt] + kSlack;
  }
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(raise) != 0, 0)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float x = max_xor32(max_xor16(mx[nt]));
      const bool up = x > st.m[nt] + kSlack;
      const float alpha = up ? __builtin_amdgcn_exp2f(st.m[nt] - x) : 1.f;   // 0 on the first visible tile
      st.m[nt] = up ? x : st.m[nt];
      st.l[nt] *= alpha;
      st.lx[nt] *= alpha;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) st.o[nt][dt] *= alpha;
    }
  }

  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  bf16x8 pop[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float muse = st.m[nt] == -INFINITY ? 0.f : st.m[nt];
    float pv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pv[i] = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][nt][i & 3], scale_log2, -muse));
    if constexpr (LSE) {
      float sx = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sx += pv[i];
      st.lx[nt] += sx;
    }
    u32x4 pw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = pack_bf16x2(pv[2 * i], pv[2 * i + 1]);
      // hidden from the compiler, which took the first pair of the operand below for all four
      asm("" : "+v"(w));
      st.l[nt] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), ones, st.l[nt], false);
      pw[i] = w;
    }
    pop[nt] = as_bf16x8(pw);
  }
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_bf16<BITS>(T.v[i][0], T.v[i][Tile<BITS>::kParts - 1], T.vs[i]);
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    const bf16x8 vt = vt_operand(v, dt);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      st.o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pop[nt], st.o[nt][dt], 0, 0, 0);
  }
}

// The same value, of which the compiler knows nothing: what is computed from it is computed where it stands, not kept
// in registers over the loops around (or before) it.
__device__ inline int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Keys of sequence s's units, and its length.
__device__ inline int unit_keys(const QAttnParams& p, int s, int& L) {
  L = seq_len(p.kv, s);
  if (!p.idx) return L;
  const int n = p.nsel[s];
  return n < 0 || L == 0 ? 0 : (n > p.ld_idx ? p.ld_idx : n);   // an empty cache has no row to stand in for absent ones
}
// Tiles of a unit (an empty one has one too: its outputs have to be written), and its length in the stream.
__device__ inline int unit_tiles(int n) { return n > 0 ? (int)(((int64_t)n + kTile - 1) / kTile) : 1; }
__device__ inline int unit_span(int n) { const int t = unit_tiles(n); return t > kMinSpan ? t : kMinSpan; }

// Shares that a unit of t tiles has of its own (t = 0: no unit), of about c tiles each.  Whatever the rounding of the
// products gives lies in [1, t], and is the same in every workgroup.
__device__ inline int own_shares(int t, int c) {
  const int k = (int)(((float)t - 0.5f) * __builtin_amdgcn_rcpf((float)c)) + 1;
  return t < kWhole ? (t > 0 ? 1 : 0) : k;
}

// Inclusive sums over the lanes.
template <int CTRL, int ROWMASK>
__device__ inline int add_dpp(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWMASK, 0xF, false); }
__device__ inline int wave_scan(int x) {
  x = add_dpp<0x111, 0xF>(x);    // row_shr 1, 2, 4, 8: within 16 lanes
  x = add_dpp<0x112, 0xF>(x);
  x = add_dpp<0x114, 0xF>(x);
  x = add_dpp<0x118, 0xF>(x);
  x = add_dpp<0x142, 0xA>(x);    // the last lane of a row of 16 to the next row (rows 1 and 3)
  return add_dpp<0x143, 0xC>(x); // lane 31 to rows 2 and 3
}

// Every kernel argument requested at entry, so that they cost one round trip to the memory that holds them rather
// than one per line where first used (attn.hip's fetch_args says more); returns 0.  Left to the compiler, the lines
// past the first came one after the other, XCD after XCD: a workgroup began its loads 2 to 15 us after its start
// (8 heads of one 8K sequence, 26.7 us).
__device__ inline int fetch_args(const QAttnParams& p) {
  int z0, z1, z2;
  asm("s_mov_b32 %0, 0" : "=s"(z0) : "s"(p.kv.k), "s"(p.kv.v), "s"(p.kv.k_scale), "s"(p.kv.v_scale), "s"(p.kv.seq_lens),
      "s"(p.kv.page_table), "s"(p.kv.stride_seq), "s"(p.kv.stride_head), "s"(p.kv.stride_tok));
  asm("s_mov_b32 %0, 0" : "=s"(z1) : "s"(z0), "s"(p.kv.stride_page), "s"(p.kv.max_seq_len), "s"(p.kv.page_size),
      "s"(p.kv.max_pages_per_seq), "s"(p.kv.num_pages), "s"(p.q), "s"(p.out), "s"(p.lse), "s"(p.idx), "s"(p.nsel));
  asm("s_mov_b32 %0, 0" : "=s"(z2) : "s"(z1), "s"(p.ld_idx), "s"(p.S), "s"(p.Hkv), "s"(p.Hq), "s"(p.G), "s"(p.nq),
      "s"(p.R), "s"(p.n_rb), "s"(p.nW), "s"(p.scale_log2), "s"(p.part), "s"(p.part_bytes),
      "s"(p.counters));
  return z2;
}

template <int BITS, int NT, int ROWS, bool LSE>
__global__ __launch_bounds__(kThreads, (Config<BITS, NT, ROWS>::kPerCu)) void qattn_kernel(QAttnParams p) {
  using TL = Tile<BITS>;
  constexpr int kTab = Config<BITS, NT, ROWS>::kTab;
  constexpr int kRows = 16 * NT;
  constexpr int kRec = kRows * (4 + kD);       // floats of a record: (m, l, lx, -) per row, then the outputs
  __shared__ Smem<BITS, NT, ROWS> sm;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lr = lane & 15;
  const int block = blockIdx.x + fetch_args(p);
  const bool gather = p.idx != nullptr;

  // ---- the share: [begin, end) of the stream, its first piece in sequence s.  The stream is counted in tiles and cut
  // every `chunk` of them; or, with per > 0, each unit has shares of its own, of `per` tiles or a little less, and the
  // stream is counted in shares.  So it is where such shares are no more than kLonger tiles longer: a share that has parts of two
  // units does two prologues and two merges one after the other (22 sequences of 650 to 2602 rows, 8 heads, 28 rows,
  // 4 bits: 25.2 -> 19.3 us; 27 of 816 to 3267, 4 heads, 24 rows, 8 bits: 28.4 -> 22.6).
  int total = 0, first_w = 0, first_t = 0;     // of this lane's sequence of the first 64: its end, its units' tiles
  for (int s0 = 0; s0 < p.S; s0 += kWave) {
    int L = 0, w = 0;
    if (s0 + lane < p.S) {
      const int n = unit_keys(p, s0 + lane, L);
      w = unit_span(n) * p.Hkv;
      if (s0 == 0) first_t = unit_tiles(n);
    }
    w = wave_scan(w);
    if (s0 == 0) first_w = w;
    total += __builtin_amdgcn_readlane(w, kWave - 1);
  }
  int chunk = (total + p.nW - 1) / p.nW;
  if (chunk < kMinSpan) chunk = kMinSpan;
  int per = 0;
  if (p.S <= kWave && p.S * p.Hkv <= p.nW) {
    // the shares that two lengths give, in one word (sums below 2 nW: a unit has at most one more than its part)
    const int ends = wave_scan((own_shares(first_t, chunk) | own_shares(first_t, chunk + kLonger) << 16) * p.Hkv);
    const uint32_t sums = (uint32_t)__builtin_amdgcn_readlane(ends, kWave - 1);
    const int part = (sums & 0xFFFFu) <= (uint32_t)p.nW ? 0 : 16;
    if ((sums >> part & 0xFFFFu) <= (uint32_t)p.nW) {
      per = part ? chunk + kLonger : chunk;
      first_w = (int)((uint32_t)ends >> part & 0xFFFFu);
      total = (int)(sums >> part & 0xFFFFu);
      chunk = 1;
    }
  }
  // the workgroups that have a share are the first of the launch, spread evenly over the XCDs
  const int working = (total + chunk - 1) / chunk * p.n_rb;
  if (block >= working) return;
  const int bid = xcd_remap(block, working);
  const int share = bid / p.n_rb, rb = bid - share * p.n_rb;
  const int begin = share * chunk;
  const int end = total - begin < chunk ? total : begin + chunk;
  int s = 0, before = 0;                       // tiles of the sequences before s
  for (int s0 = 0, acc = 0; s0 < p.S; s0 += kWave) {
    int w = first_w;
    if (s0 > 0) {
      int L = 0;
      w = 0;
      if (s0 + lane < p.S) w = unit_span(unit_keys(p, s0 + lane, L)) * p.Hkv;
      w = wave_scan(w);
    }
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(acc + w <= begin));
    if (c < kWave) {
      s = s0 + c;
      before = acc + (c > 0 ? __builtin_amdgcn_readlane(w, c - 1) : 0);
      break;
    }
    acc += __builtin_amdgcn_readlane(w, kWave - 1);
  }
  s = __builtin_amdgcn_readfirstlane(s);
  before = __builtin_amdgcn_readfirstlane(before);

  int L, n = __builtin_amdgcn_readfirstlane(unit_keys(p, s, L));
  L = __builtin_amdgcn_readfirstlane(L);
  int T = unit_tiles(n), span = per == 0 ? unit_span(n) : own_shares(T, per);
  int g = (begin - before) / span;
  int unit0 = before + g * span;               // where the unit begins in the stream

  const uint32_t ring_lds = lds_addr(&sm.u.ring[wave][0][0]);
  const uint32_t tok = (uint32_t)p.kv.stride_tok, tok_bytes = tok * (uint32_t)TL::kRow;   // 15 rows below 2^31: host-checked
  uint32_t k_off[TL::kParts], v_off[TL::kParts];           // this lane's bytes of a whole sub-tile's loads
#pragma unroll
  for (int e = 0; e < TL::kParts; ++e) {
    k_off[e] = (uint32_t)TL::k_row(lane, e) * tok_bytes + 16u * (uint32_t)TL::k_chunk(lane, e);
    v_off[e] = (uint32_t)TL::v_row(lane, e) * tok_bytes + 16u * (uint32_t)TL::v_chunk(lane);
  }

  // whether the share has a piece of the unit
  auto taken = [&] { return per > 0 || T >= kWhole || (begin - unit0 < (span + 1) / 2 && end - unit0 >= (span + 1) / 2); };
  // to the next unit; false where the share ends (with per > 0 it always does)
  auto advance = [&] {
    unit0 += span;
    if (unit0 >= end) return false;
    if (++g == p.Hkv) {
      g = 0;
      ++s;
      n = __builtin_amdgcn_readfirstlane(unit_keys(p, s, L));
      L = __builtin_amdgcn_readfirstlane(L);
      T = unit_tiles(n);
      span = unit_span(n);
    }
    return true;
  };
  while (!taken())
    if (!advance()) return;

  for (;;) {   // ---- one piece: tiles [t0, t1) of unit (s, g)
    const bool whole = T < kWhole;
    int t0 = whole || begin <= unit0 ? 0 : begin - unit0;
    int t1 = whole || T <= end - unit0 ? T : end - unit0;
    if (per > 0 && !whole) {   // the share's part of T tiles, cut evenly
      const int j = begin - unit0, q = T / span, more = T - q * span;
      t0 = j * q + (j < more ? j : more);
      t1 = t0 + q + (j < more ? 1 : 0);
    }
    const int tn = (n + kTile - 1) / kTile < t1 ? (n + kTile - 1) / kTile : t1;   // tiles that hold keys

    const int lane_q = here(lane), lgq = lane_q >> 4, lrq = lane_q & 15;
    RowState<NT> st;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      st.m[nt] = -INFINITY;
      st.l[nt] = st.lx[nt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) st.o[nt][dt] = zero4();
    }
    // each row's position: selected entries lie below the length, and the one query at its end sees them all
    if (lane_q < 4 * NT) {
      const int r = 4 * NT * wave + lane_q, row = rb * kRows + r;
      sm.rowpos[r] = row < p.R && !gather ? L - p.nq + row / p.G : 0x7FFFFFFF;
    }
    // query rows to LDS, four a load; rows past the last one repeat it
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const int r0 = 4 * (NT * wave + k), r = r0 + lgq;
      const int row = rb * kRows + r < p.R ? rb * kRows + r : p.R - 1;
      const int j = row / p.G;
      dma16_hidden(p.q + (((int64_t)s * p.nq + j) * p.Hq + g * p.G + (row - j * p.G)) * kD + 8 * (lrq ^ k_swizzle(r & 15)),
                   lds_addr(&sm.r.q[r0][0]));
    }
    if (tid < kBlocks) sm.nan_from[tid] = 0x7FFFFFFF;
    const int minpos = gather ? 0x7FFFFFFF : L - p.nq + rb * kRows / p.G;         // position of the block's first row
    const uint32_t head_row = (uint32_t)((int64_t)s * p.kv.stride_seq + (int64_t)g * p.kv.stride_head);

    for (int c0 = t0; c0 < tn;) {   // ---- as many tiles as the table covers
      int c1 = tn;
      // tiles from first_dirty on may hold keys that are absent or hidden from some row
      int first_dirty = n / kTile;
      if (!gather && (minpos + 1) / kTile < first_dirty) first_dirty = minpos < 0 ? 0 : (minpos + 1) / kTile;
      bool holes = false;            // some page that the table covers is outside the pool
      if constexpr (ROWS == kQPages) {
        // one entry per sub-tile: the row of its first key
        if (c1 - c0 > kTab / 2) c1 = c0 + kTab / 2;
        const int32_t* prow = p.kv.page_table + (int64_t)s * p.kv.max_pages_per_seq;
        int bad = 0;
        for (int j = tid; j < 2 * (c1 - c0); j += kThreads) {
          const int t = c0 * kTile + 16 * j;
          uint32_t x = kAbsent;
          if (t < n) {
            const int pi = t / p.kv.page_size, pg = prow[pi];
            if ((unsigned)pg < (unsigned)p.kv.num_pages)
              x = (uint32_t)((int64_t)pg * p.kv.stride_page + (int64_t)g * p.kv.stride_head + (int64_t)(t - pi * p.kv.page_size) * tok);
            else bad = 1;
          }
          sm.tab[j] = x;
        }
        holes = __builtin_amdgcn_readfirstlane(__syncthreads_or(bad)) != 0;
        if (holes) first_dirty = c0;
      } else if constexpr (ROWS == kQTable) {
        if (c1 - c0 > kTab / kTile) c1 = c0 + kTab / kTile;
        const int32_t* list = gather ? p.idx + ((int64_t)s * p.Hkv + g) * p.ld_idx : nullptr;
        if (tid == 0) sm.first_hole = 0x7FFFFFFF;
        __syncthreads();
        for (int i = tid; i < (c1 - c0) * kTile; i += kThreads) {
          const int e = c0 * kTile + i;
          int t = -1;
          if (e < n) t = list ? list[e] : e;
          int64_t row = -1;
          if (t >= 0 && t < L) {
            row = row_of(p.kv, s, t);
            if (row >= 0) row += (int64_t)g * p.kv.stride_head;
          }
          sm.tab[i] = row >= 0 ? (uint32_t)row : kAbsent;
          if (row < 0) atomicMin(&sm.first_hole, c0 + i / kTile);
        }
        __syncthreads();
        const int hole = __builtin_amdgcn_readfirstlane(sm.first_hole);
        if (hole < first_dirty) first_dirty = hole;
      }

      // rows of a tile's sub-tiles, their first keys' (uniform), and the last row of each that may be read
      struct Where { uint32_t row[2]; int lim[2]; };
      auto where = [&](int c) {
        Where at{{0u, 0u}, {15, 15}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int t = c * kTile + 16 * h;
          if constexpr (ROWS == kQContiguous) {
            if (t + 15 >= n) at.lim[h] = t < n ? n - 1 - t : 0;
            at.row[h] = head_row + (uint32_t)(t < n ? t : n - 1) * tok;
          } else if constexpr (ROWS == kQPages) {
            const uint32_t x = (uint32_t)__builtin_amdgcn_readfirstlane((int)sm.tab[2 * (c - c0) + h]);
            at.row[h] = x == kAbsent ? 0u : x;             // past the keys, or absent: any row
          }
        }
        return at;
      };
      // Direct loads of tile c into ring slot `slot`, non-temporal: a call reads each row once, or once a row block and
      // that at the same time, and the next reader of a layer's cache comes after the other layers'.  Selected rows,
      // non-temporal and not: 64 heads of 8 bits in pages, 100 and 118 us; 1024 of 4K-8K rows, 32 x 64 heads of 4 bits,
      // 68 and 78 us; 512 of them 42 and 47 us (where the caches still hold the rows of the call before, 42 and 40).
      auto issue = [&](int c, int slot, const Where& at) {
        const uint32_t dst = ring_lds + (uint32_t)(slot * TL::kBytes);
        if constexpr (ROWS == kQTable) {
          const uint32_t* tab = sm.tab + (c - c0) * kTile;
          auto row_at = [&](int r) { const uint32_t x = tab[r]; return x == kAbsent ? 0u : x; };
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < TL::kParts; ++e) {
              const uint32_t to = dst + 1024u * (uint32_t)(TL::kParts * h + e);
              const uint8_t* kp = p.kv.k + (uint64_t)row_at(16 * h + TL::k_row(lane, e)) * TL::kRow + 16 * TL::k_chunk(lane, e);
              const uint8_t* vp = p.kv.v + (uint64_t)row_at(16 * h + TL::v_row(lane, e)) * TL::kRow + 16 * TL::v_chunk(lane);
              dma16_nt_hidden(reinterpret_cast<const uint16_t*>(kp), to);
              dma16_nt_hidden(reinterpret_cast<const uint16_t*>(vp), to + TL::kV);
            }
          dma4_hidden((lane < kTile ? p.kv.k_scale : p.kv.v_scale) + (uint64_t)row_at(lane & 31) * kBlocks, dst + TL::kS);
        } else {
          const uint32_t row0 = at.row[0], row1 = at.row[1];
          const int lim0 = at.lim[0], lim1 = at.lim[1];
          auto loads = [&](auto whole_tag) {
            constexpr bool WHOLE = decltype(whole_tag)::value;
            const int lane_i = WHOLE ? lane : here(lane);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint8_t* kb = p.kv.k + (uint64_t)(h ? row1 : row0) * TL::kRow;
              const uint8_t* vb = p.kv.v + (uint64_t)(h ? row1 : row0) * TL::kRow;
#pragma unroll
              for (int e = 0; e < TL::kParts; ++e) {
                const uint32_t to = dst + 1024u * (uint32_t)(TL::kParts * h + e);
                uint32_t ko = k_off[e], vo = v_off[e];
                if (!WHOLE) {
                  const int lim = h ? lim1 : lim0;
                  const int kr = TL::k_row(lane_i, e) < lim ? TL::k_row(lane_i, e) : lim;
                  const int vr = TL::v_row(lane_i, e) < lim ? TL::v_row(lane_i, e) : lim;
                  ko = (uint32_t)kr * tok_bytes + 16u * (uint32_t)TL::k_chunk(lane_i, e);
                  vo = (uint32_t)vr * tok_bytes + 16u * (uint32_t)TL::v_chunk(lane_i);
                }
                dma16_nt_hidden(reinterpret_cast<const uint16_t*>(kb), ko, to);
                dma16_nt_hidden(reinterpret_cast<const uint16_t*>(vb), vo, to + TL::kV);
              }
            }
            const int lane_s = here(lane);                 // three instructions a tile rather than three registers
            const bool upper = (lane_s & 16) != 0;
            int sr = lane_s & 15;
            if (!WHOLE) sr = sr < (upper ? lim1 : lim0) ? sr : (upper ? lim1 : lim0);
            const uint8_t* sb = lane_s < kTile ? p.kv.k_scale : p.kv.v_scale;
            dma4_hidden(sb + (uint64_t)((upper ? row1 : row0) + (uint32_t)sr * tok) * kBlocks, dst + TL::kS);
          };
          if (ROWS == kQPages || c * kTile + kTile <= n) loads(BoolTag<true>{});
          else loads(BoolTag<false>{});
        }
      };

      const int mine = c1 - c0 > wave ? (c1 - c0 - wave + kWaves - 1) / kWaves : 0;   // tiles of this wave
      for (int i = 0; i < kRing && i < mine; ++i) issue(c0 + wave + i * kWaves, i, where(c0 + wave + i * kWaves));
      if (c0 == t0) {
        // the query rows, which were asked for first, and every load and store before them
        if (mine >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * TL::kLoads) : "memory");
        else if (mine == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TL::kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      // The second workgroup of a CU runs its first half at a raised priority: issue prefers the older waves, which
      // would be done early and leave the younger ones alone, one a SIMD (16K x 8 in 4 bits 41.0 -> 39.0 us, 8 bits
      // 54.7 -> 53.0; raised throughout 40.0 and 53.7).
      if (blockIdx.x >= kCus) __builtin_amdgcn_s_setprio(1);
      int i = 0, slot = 0;
      // tile i of this wave: its codes to registers, its slot filled again, the products
      auto step = [&](auto dirty_tag) {
        constexpr bool DIRTY = decltype(dirty_tag)::value;
        const int c = c0 + wave + i * kWaves;
        if (i + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TL::kLoads) : "memory");   // the next tile is on its way
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (2 * i == mine || 2 * i == mine - 1) __builtin_amdgcn_s_setprio(0);
        const bool more = i + kRing < mine;
        const Where next = where(more ? c + kRing * kWaves : c);
        TileRegs<BITS> tile;
        read_tile<BITS>(tile, sm.u.ring[wave][slot], lane);
        // key slot 4h + j of this lane: key c*32 + 16h + 4*lg + j
        const int key0 = c * kTile + 4 * lg;
        uint32_t there = 0xFFu;
        if constexpr (DIRTY) {
          if constexpr (ROWS == kQTable) {
            const uint32_t ok = ~(uint32_t)__builtin_amdgcn_ballot_w64(sm.tab[(c - c0) * kTile + (lane & 31)] == kAbsent) >> (4 * lg);
            there = (ok & 0xFu) | ((ok >> 12) & 0xF0u);
          } else {
            there = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) there |= key0 + 16 * (j >> 2) + (j & 3) < n ? 1u << j : 0u;
            if constexpr (ROWS == kQPages) {
              if (holes) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  if (sm.tab[2 * (c - c0) + h] == kAbsent) there &= h ? 0x0Fu : 0xF0u;
              }
            }
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read: it may be filled again
        if (more) issue(c + kRing * kWaves, slot, next);
        tile_step<BITS, NT, DIRTY, LSE>(st, tile, sm.r.q, p.scale_log2, there, key0, lane, sm.rowpos, sm.nan_from);
        ++i;
        slot ^= 1;
      };
      // in loops of their own: as two branches of one, the accumulators were copied at every tile
      const int clean = first_dirty > c0 + wave ? (first_dirty - c0 - wave + kWaves - 1) / kWaves : 0;
      while (i < mine && i < clean) step(BoolTag<false>{});
      while (i < mine) step(BoolTag<true>{});
      __builtin_amdgcn_s_setprio(0);
      c0 = c1;
      if (ROWS != kQContiguous && c0 < tn) __syncthreads();   // the table is filled again
    }

    // ---- the four waves' states, through LDS, kPart row tiles at a time.  Thread -> row r of a part and the kPer
    // outputs from d0 on
    constexpr int kPart = Config<BITS, NT, ROWS>::kPart, kParts = NT / kPart, kPartRows = 16 * kPart;
    constexpr int kPer = kPartRows * kD / kThreads;        // 8 or 16
    const int tid_m = here(tid), lgm = (tid_m >> 4) & 3, lrm = tid_m & 15;
    const int r = tid_m / (kD / kPer), d0 = (tid_m % (kD / kPer)) * kPer;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the query rows of a piece without keys
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float l = st.l[nt], lx = st.lx[nt];
      l += shfl_xor_f(l, 16);
      l += shfl_xor_f(l, 32);
      if constexpr (LSE) {
        lx += shfl_xor_f(lx, 16);
        lx += shfl_xor_f(lx, 32);
      }
      if (lgm == 0) {
        sm.r.stat.m[wave][16 * nt + lrm] = st.m[nt];
        sm.r.stat.l[wave][16 * nt + lrm] = l;
        sm.r.stat.lx[wave][16 * nt + lrm] = lx;
      }
    }
    float M[kParts], Ls[kParts], Lx[kParts], acc[kParts][kPer];
#pragma unroll
    for (int pt = 0; pt < kParts; ++pt) {
      if (pt > 0) __syncthreads();                         // the part before is read
#pragma unroll
      for (int n1 = 0; n1 < kPart; ++n1) {
        const int nt = pt * kPart + n1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* dst = &sm.u.o[wave][16 * n1 + lrm][32 * lgm + 8 * i];
          *reinterpret_cast<f32x4*>(dst) = f32x4{st.o[nt][0][i], st.o[nt][1][i], st.o[nt][2][i], st.o[nt][3][i]};
          *reinterpret_cast<f32x4*>(dst + 4) = f32x4{st.o[nt][4][i], st.o[nt][5][i], st.o[nt][6][i], st.o[nt][7][i]};
        }
      }
      __syncthreads();
      const int rr = pt * kPartRows + r;
      M[pt] = -INFINITY;
      Ls[pt] = Lx[pt] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M[pt] = fmaxf(M[pt], sm.r.stat.m[w][rr]);
      const float Mu = M[pt] == -INFINITY ? 0.f : M[pt];
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[pt][e] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float wt = exp2f(sm.r.stat.m[w][rr] - Mu);
        Ls[pt] += wt * sm.r.stat.l[w][rr];
        if constexpr (LSE) Lx[pt] += wt * sm.r.stat.lx[w][rr];
#pragma unroll
        for (int e = 0; e < kPer; e += 4) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(&sm.u.o[w][r][d0 + e]);
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[pt][e + k] += wt * x[k];
        }
      }
      if (sm.nan_from[d0 >> 5] <= (gather ? 0x7FFFFFFE : L - p.nq + (rb * kRows + rr) / p.G)) {   // a thread's outputs lie in one block
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[pt][e] = __uint_as_float(0x7FC00000u);
      }
    }
    auto row_valid = [&](int pt) { return rb * kRows + pt * kPartRows + r < p.R; };
    auto write_final = [&](int pt, float Mf, float Lf, float Lxf, const float (&a)[kPer]) {
      if (!row_valid(pt)) return;
      const int row = rb * kRows + pt * kPartRows + r, jrow = row / p.G;
      const int64_t orow = ((int64_t)s * p.nq + jrow) * p.Hq + g * p.G + (row - jrow * p.G);
      const float inv = Lf == 0.f ? 0.f : 1.f / Lf;        // no visible key: 0
      uint16_t* dst = p.out + orow * kD + d0;
#pragma unroll
      for (int e = 0; e < kPer; e += 8)
        *reinterpret_cast<u32x4*>(dst + e) =
            u32x4{pack_bf16x2(a[e] * inv, a[e + 1] * inv), pack_bf16x2(a[e + 2] * inv, a[e + 3] * inv),
                  pack_bf16x2(a[e + 4] * inv, a[e + 5] * inv), pack_bf16x2(a[e + 6] * inv, a[e + 7] * inv)};
      if (LSE && d0 == 0) p.lse[orow] = Lxf == 0.f ? -INFINITY : (Mf + __log2f(Lxf)) * kLn2;
    };

    // ---- pieces of the unit: shares w0 .. w1
    const int w0 = unit0 / chunk, w1 = (unit0 + span - 1) / chunk;
    if (whole || w0 == w1) {
#pragma unroll
      for (int pt = 0; pt < kParts; ++pt) write_final(pt, M[pt], Ls[pt], Lx[pt], acc[pt]);
    } else {
      const __amdgpu_buffer_rsrc_t rec = make_rsrc(p.part, p.part_bytes);
      // a share leaves at most two records: of a unit that began before it, and of one that goes on after it
      auto at = [&](int w) { return (uint32_t)(2 * (w * p.n_rb + rb) + (w == w0 ? 1 : 0)) * (uint32_t)(kRec * 4); };
      auto store = [&](int pt, int w, float Mr, float Lr, float Lxr, const float (&a)[kPer]) {
        if (!row_valid(pt)) return;
        if (d0 == 0) store16_coherent(rec, at(w) + 16 * (pt * kPartRows + r), f32x4{Mr, Lr, Lxr, 0.f});
#pragma unroll
        for (int c = 0; c < kPer / 4; ++c)
          store16_coherent(rec, at(w) + 16 * kRows + 16 * ((pt * (kPer / 4) + c) * kThreads + tid_m),
                           f32x4{a[4 * c], a[4 * c + 1], a[4 * c + 2], a[4 * c + 3]});
      };
      float Mg, Lg, Lxg, ag[kPer];
      // records of shares first, first + step, ..., in that order, a batch of loads at a time
      auto merge = [&](int pt, int first, int count, int step) {
        Mg = -INFINITY;
        Lg = Lxg = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) ag[e] = 0.f;
        if (!row_valid(pt)) return;
        constexpr int kBatch = kPer == 8 ? 8 : 4;            // all loads of a batch are issued before any is used
        for (int k0 = 0; k0 < count; k0 += kBatch) {
          f32x4 sv[kBatch], ov[kBatch][kPer / 4];
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            // past the last record: an address past the buffer, which reads as zeros
            const uint32_t a = k0 + u < count ? at(first + (k0 + u) * step) : p.part_bytes;
            sv[u] = load16_coherent(rec, a + 16 * (pt * kPartRows + r));
#pragma unroll
            for (int c = 0; c < kPer / 4; ++c)
              ov[u][c] = load16_coherent(rec, a + 16 * kRows + 16 * ((pt * (kPer / 4) + c) * kThreads + tid_m));
          }
          float mb = Mg;
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            sv[u][0] = k0 + u < count ? sv[u][0] : -INFINITY;
            mb = fmaxf(mb, sv[u][0]);
          }
          const float mbu = mb == -INFINITY ? 0.f : mb;
          const float sc = exp2f(Mg - mbu);
          Lg *= sc;
          Lxg *= sc;
#pragma unroll
          for (int e = 0; e < kPer; ++e) ag[e] *= sc;
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const float w = exp2f(sv[u][0] - mbu);
            Lg += w * sv[u][1];
            Lxg += w * sv[u][2];
#pragma unroll
            for (int c = 0; c < kPer / 4; ++c)
#pragma unroll
              for (int k = 0; k < 4; ++k) ag[4 * c + k] += w * ov[u][c][k];
          }
          Mg = mb;
        }
      };
      // true in the workgroup that arrives last of `count` at the line of share w
      auto last_of = [&](int line, int count) {
        wait_vmem();
        __syncthreads();
        if (tid == 0) {
          uint32_t* ctr = counter_line(p.counters, line);
          const bool last = arrive(ctr, (uint32_t)count);
          if (last) reset_counter(ctr);                    // ready for the next call
          sm.last = last;
        }
        __syncthreads();
        return sm.last != 0;
      };
      const int np = w1 - w0 + 1;
      const bool two = np > kGroup;
      const int grp = (share - w0) / kGroup;
      const int g0 = two ? w0 + grp * kGroup : w0;
      const int gn = two ? (np - grp * kGroup < kGroup ? np - grp * kGroup : kGroup) : np;
#pragma unroll
      for (int pt = 0; pt < kParts; ++pt) store(pt, share, M[pt], Ls[pt], Lx[pt], acc[pt]);
      // counter lines, each shares x row blocks: whole units, named by their first share; first groups, by the same;
      // other groups, by theirs, in which another unit's first group may begin
      const int region = !two ? 0 : grp == 0 ? 1 : 2;
      if (last_of((region * p.nW + g0) * p.n_rb + rb, gn)) {
        for (int pt = 0; pt < kParts; ++pt) {
          merge(pt, g0, gn, 1);
          if (!two) {
            write_final(pt, Mg, Lg, Lxg, ag);
          } else {
            __syncthreads();                               // the group's first record is read: it is written again
            store(pt, g0, Mg, Lg, Lxg, ag);
          }
        }
        if (two && last_of(w0 * p.n_rb + rb, (np + kGroup - 1) / kGroup)) {
          for (int pt = 0; pt < kParts; ++pt) {
            merge(pt, w0, (np + kGroup - 1) / kGroup, kGroup);
            write_final(pt, Mg, Lg, Lxg, ag);
          }
        }
      }
    }

    do {
      if (!advance()) return;
    } while (!taken());
    __syncthreads();   // the merge buffer is read: the ring may be filled again
  }
}

template <int BITS, int NT, bool LSE>
hipError_t launch_rows(const QAttnParams& p, const QAttnPlan& pl, hipStream_t stream) {
  const dim3 grid((unsigned)pl.nblk), block(kThreads);
  if (pl.rows == kQContiguous) hipLaunchKernelGGL((qattn_kernel<BITS, NT, kQContiguous, LSE>), grid, block, 0, stream, p);
  else if (pl.rows == kQPages) hipLaunchKernelGGL((qattn_kernel<BITS, NT, kQPages, LSE>), grid, block, 0, stream, p);
  else if constexpr (NT < 3) hipLaunchKernelGGL((qattn_kernel<BITS, NT, kQTable, LSE>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template <int BITS>
hipError_t launch_bits(const QAttnParams& p, const QAttnPlan& pl, hipStream_t stream) {
  if (pl.nt == 1) return p.lse ? launch_rows<BITS, 1, true>(p, pl, stream) : launch_rows<BITS, 1, false>(p, pl, stream);
  if (pl.nt == 2) return p.lse ? launch_rows<BITS, 2, true>(p, pl, stream) : launch_rows<BITS, 2, false>(p, pl, stream);
  return p.lse ? launch_rows<BITS, 3, true>(p, pl, stream) : launch_rows<BITS, 3, false>(p, pl, stream);
}

}  // namespace

QAttnPlan plan_qattn(int S, int Hkv, int Hq, int nq, int64_t entries, bool gather, bool paged, int page_size) {
  QAttnPlan pl{};
  const int64_t R = (int64_t)nq * (Hq / Hkv);
  pl.R = (int)(R < (1 << 30) ? R : (1 << 30));
  pl.rows = gather ? kQTable : !paged ? kQContiguous : page_size % 16 == 0 ? kQPages : kQTable;
  const int64_t span = (entries + kTile - 1) / kTile;
  const int64_t tiles = (int64_t)S * Hkv * (span > kMinSpan ? span : kMinSpan);
  // Blocks of 48 rows where they are fewer by more than a quarter (their turns take about 4/3 as long) and the stream is
  // long enough for their longer merges.  With 48 and 32, 4 bits: 36 rows, 8 x 8 heads of 16K, 48 and 57 us (8 bits 58
  // and 70); 72 rows 71 and 80; 48 rows, 16 x 8 of 1K to 4K, 29 and 32; but 45 rows, 3 x 8 of 12.5K, 33 and 29.
  const bool three = pl.rows != kQTable && 4 * ((R + 47) / 48) < 3 * ((R + 31) / 32) && tiles >= 24 * kMaxBlocks;
  pl.nt = R <= 16 ? 1 : three ? 3 : 2;
  pl.n_rb = (pl.R + 16 * pl.nt - 1) / (16 * pl.nt);
  int64_t nW = (int64_t)S * Hkv * (((span > kMinSpan ? span : kMinSpan) + kMinSpan - 1) / kMinSpan);   // whole shares a unit
  const int64_t most = kMaxBlocks / pl.n_rb > 1 ? kMaxBlocks / pl.n_rb : 1;
  if (nW > most) nW = most;
  pl.nW = (int)nW;
  pl.nblk = tiles > (1 << 30) || entries > (1 << 30) || nW * pl.n_rb >= (1 << 22) ? -1 : nW * pl.n_rb;
  pl.counter_bytes = BD_WS_COUNTER_BYTES;
  const size_t rec = sizeof(float) * 16 * pl.nt * (4 + kD);
  pl.record_bytes = nW > 1 && pl.nblk > 0 ? align256(2 * rec * (size_t)pl.nblk) : 0;
  pl.ws_bytes = pl.counter_bytes + pl.record_bytes;
  return pl;
}

hipError_t launch_qattn(const QAttnParams& p, const QAttnPlan& pl, int bits, hipStream_t stream) {
  return bits == 4 ? launch_bits<4>(p, pl, stream) : launch_bits<8>(p, pl, stream);
}

}  // namespace bd
