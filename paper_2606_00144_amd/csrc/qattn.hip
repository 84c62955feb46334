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
// row.  A wave streams its tiles through a ring in LDS of its own with direct loads, so that about 100 KiB a CU are
// on their way while 4 waves (two workgroups a CU) convert and multiply.
//
// Work decomposition.  All (sequence, KV head) units' tiles form one stream, which is cut into nW equal shares from
// the lengths on the device; workgroup (share, row block) takes the units that its share meets, one after the
// other.  A share's time depends on the lengths as they are, not on the capacity or on the longest sequence.  A
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
constexpr int kTab = 2048;                     // table entries (rows, or pages)
constexpr int kGroup = 8;                      // records merged by one batch of loads
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;                  // lazy-rescale headroom, log2 units
constexpr uint32_t kAbsent = 0xFFFFFFFFu;
constexpr int kMaxBlocks = 512;                // workgroups of a launch: two per CU

// A tile in LDS: K's codes, V's codes, then the 32 scale words of K and of V.
template <int BITS>
struct Tile {
  static constexpr int kRow = QFormat<BITS>::kRow;
  static constexpr int kParts = kRow / 64;               // 1 KiB loads per 16 rows of K or V
  static constexpr int kLoads = 4 * kParts + 1;          // loads of a tile
  static constexpr int kV = kTile * kRow, kS = 2 * kV, kBytes = kS + 2 * kTile * kBlocks;
  static constexpr int kRing = BITS == 4 ? 4 : 2;

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

template <int BITS, int NT>
struct Smem {
  alignas(16) uint32_t tab[kTab];
  union {
    alignas(64) uint8_t ring[kWaves][Tile<BITS>::kRing][Tile<BITS>::kBytes];
    struct {
      alignas(16) float o[kWaves][16 * NT][kD + 4];
      float m[kWaves][16 * NT], l[kWaves][16 * NT], lx[kWaves][16 * NT];
    } merge;
  } u;
  int32_t last;
};

template <int NT>
struct RowState {
  f32x4 o[NT][8];     // O^T[d-tile][row tile]: register i of d-tile dt holds d = 32*(l/16) + 8*i + dt
  f32x4 l[NT];        // sums of the rounded weights (every register holds the row's)
  float m[NT];        // reference maximum (log2 domain)
  float lx[NT];       // this lane's sum of the unrounded weights (log-sum-exp only)
};

__device__ inline f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ inline uint32_t as_word(const __attribute__((ext_vector_type(2))) __bf16& v) { return __builtin_bit_cast(uint32_t, v); }

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

// One tile of one wave.  `dirty` (uniform): some key of the tile is absent or hidden from some row; key slot i of
// this lane is absent unless bit i of `there`, and lies at position pos0 + 16*(i/4) + i%4.
template <int BITS, int NT>
__device__ inline void tile_step(RowState<NT>& st, TileRegs<BITS>& T, const bf16x8 (&qop)[NT][4], const int (&rowpos)[NT],
                                 float scale_log2, bool dirty, uint32_t there, int pos0, bool want_lx) {
  f32x4 sc[2][NT];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    bf16x8 kop[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BITS == 4) kop[j] = as_bf16x8(to_bf16<4>(T.k[h][0][j], 0u, T.ks[h]));
      else kop[j] = as_bf16x8(to_bf16<8>(T.k[h][j >> 1][2 * (j & 1)], T.k[h][j >> 1][2 * (j & 1) + 1], T.ks[h]));
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      f32x4 a = zero4();
#pragma unroll
      for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[j], qop[nt][j], a, 0, 0, 0);
      sc[h][nt] = a;
    }
  }
  if (dirty) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool present = (there >> i) & 1u;
      const int pos = pos0 + 16 * (i >> 2) + (i & 3);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        if (!(present && pos <= rowpos[nt])) sc[i >> 2][nt][i & 3] = -INFINITY;
      // what lies in absent rows (stale memory) must not reach the products: 0 * NaN
#pragma unroll
      for (int e = 0; e < Tile<BITS>::kParts; ++e) T.v[i][e] = present ? T.v[i][e] : 0u;
      T.vs[i] = present ? T.vs[i] : 0x3F800000u;
    }
  }

  float mx[NT];
  bool raise = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float v = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = fmaxf(v, sc[i >> 2][nt][i & 3]);
    mx[nt] = max_xor32(max_xor16(v)) * scale_log2;    // scale > 0: the max commutes with it
    raise |= mx[nt] > st.m[nt] + kSlack;
  }
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(raise) != 0, 0)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const bool up = mx[nt] > st.m[nt] + kSlack;
      const float alpha = up ? __builtin_amdgcn_exp2f(st.m[nt] - mx[nt]) : 1.f;   // 0 on the first visible tile
      st.m[nt] = up ? mx[nt] : st.m[nt];
      st.l[nt] *= alpha;
      st.lx[nt] *= alpha;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) st.o[nt][dt] *= alpha;
    }
  }

  const bf16x8 ones = as_bf16x8(u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
  bf16x8 pop[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float muse = st.m[nt] == -INFINITY ? 0.f : st.m[nt];
    float pv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pv[i] = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][nt][i & 3], scale_log2, -muse));
    u32x4 pw;
#pragma unroll
    for (int i = 0; i < 4; ++i) pw[i] = pack_bf16x2(pv[2 * i], pv[2 * i + 1]);
    pop[nt] = as_bf16x8(pw);
    if (want_lx) {
      float sx = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sx += pv[i];
      st.lx[nt] += sx;
    }
    st.l[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pop[nt], st.l[nt], 0, 0, 0);
  }

  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_bf16<BITS>(T.v[i][0], T.v[i][Tile<BITS>::kParts - 1], T.vs[i]);

  // A value that is not a number belongs only to the rows that see its key: 0 * NaN in the product would reach the
  // others.  Such values are taken out of the product and counted, per row and d, by one of ones.
  if (dirty) {
    uint32_t bad = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w)
        bad |= ((v[i][w] & 0x7F80u) == 0x7F80u || (v[i][w] & 0x7F800000u) == 0x7F800000u) ? 1u : 0u;
    if (__builtin_amdgcn_ballot_w64(bad != 0u) != 0) {
      u32x4 ind[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const bool lo = (v[i][w] & 0x7F80u) == 0x7F80u, hi = (v[i][w] & 0x7F800000u) == 0x7F800000u;
          ind[i][w] = (lo ? 0x3F80u : 0u) | (hi ? 0x3F800000u : 0u);
          v[i][w] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
        }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        u32x4 sees = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (((there >> i) & 1u) && pos0 + 16 * (i >> 2) + (i & 3) <= rowpos[nt]) sees[i >> 1] |= (i & 1) ? 0x3F800000u : 0x3F80u;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt_operand(ind, dt), as_bf16x8(sees), zero4(), 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (n[i] > 0.f) st.o[nt][dt][i] = __uint_as_float(0x7FC00000u);
        }
      }
    }
  }
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    const bf16x8 vt = vt_operand(v, dt);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      st.o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pop[nt], st.o[nt][dt], 0, 0, 0);
  }
}

// Wait until at most `tiles` tiles of this wave are still on their way.
template <int BITS>
__device__ inline void wait_tiles(int tiles) {
  constexpr int n = Tile<BITS>::kLoads;
  if (tiles >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * n) : "memory");
  else if (tiles == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * n) : "memory");
  else if (tiles == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Keys of sequence s's units, and its length.
__device__ inline int unit_keys(const QAttnParams& p, int s, int& L) {
  L = seq_len(p.kv, s);
  if (!p.idx) return L;
  const int n = p.nsel[s];
  return n < 0 || L == 0 ? 0 : (n > p.ld_idx ? p.ld_idx : n);   // an empty cache has no row to stand in for absent ones
}
// Tiles of a unit: an empty one still takes part, its outputs have to be written.
__device__ inline int unit_tiles(int n) { return n > 0 ? (int)(((int64_t)n + kTile - 1) / kTile) : 1; }

__device__ inline int wave_scan(int x, int lane) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

template <int BITS, int NT, int ROWS>
__global__ __launch_bounds__(kThreads, 2) void qattn_kernel(QAttnParams p) {
  using TL = Tile<BITS>;
  constexpr int kRows = 16 * NT;
  constexpr int kRec = kRows * (4 + kD);       // floats of a record: (m, l, lx, -) per row, then the outputs
  __shared__ Smem<BITS, NT> sm;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lr = lane & 15;
  const int bid = xcd_remap(blockIdx.x, gridDim.x);
  const int share = bid / p.n_rb, rb = bid - share * p.n_rb;
  const bool gather = p.idx != nullptr;

  // ---- the share: tiles [pos, end) of the stream, the first of them in sequence s
  int total = 0, first_w = 0;                  // first_w: this lane's sequence of the first 64, in tiles
  for (int s0 = 0; s0 < p.S; s0 += kWave) {
    int L = 0, w = 0;
    if (s0 + lane < p.S) w = unit_tiles(unit_keys(p, s0 + lane, L)) * p.Hkv;
    w = wave_scan(w, lane);
    if (s0 == 0) first_w = w;
    total += __builtin_amdgcn_readlane(w, kWave - 1);
  }
  int chunk = (total + p.nW - 1) / p.nW;
  if (chunk < p.min_share) chunk = p.min_share;
  const int64_t pos64 = (int64_t)share * chunk;
  if (pos64 >= total) return;
  int pos = (int)pos64;
  const int end = total - pos < chunk ? total : pos + chunk;
  int s = 0, before = 0;                       // tiles of the sequences before s
  for (int s0 = 0, acc = 0; s0 < p.S; s0 += kWave) {
    int w = first_w;
    if (s0 > 0) {
      int L = 0;
      w = 0;
      if (s0 + lane < p.S) w = unit_tiles(unit_keys(p, s0 + lane, L)) * p.Hkv;
      w = wave_scan(w, lane);
    }
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(acc + w <= pos));
    if (c < kWave) {
      s = s0 + c;
      before = acc + (c > 0 ? __builtin_amdgcn_readlane(w, c - 1) : 0);
      break;
    }
    acc += __builtin_amdgcn_readlane(w, kWave - 1);
  }
  s = __builtin_amdgcn_readfirstlane(s);
  before = __builtin_amdgcn_readfirstlane(before);

  int L, n = unit_keys(p, s, L);
  int T = unit_tiles(n);
  int g = (pos - before) / T;
  int unit0 = before + g * T;                  // the unit's first tile in the stream

  const uint32_t ring_lds = lds_addr(&sm.u.ring[wave][0][0]);
  const uint32_t tok = (uint32_t)p.kv.stride_tok, tok_bytes = tok * (uint32_t)TL::kRow;   // 15 rows below 2^31: host-checked
  const uint8_t* const scales = lane < kTile ? p.kv.k_scale : p.kv.v_scale;
  const bool want_lx = p.lse != nullptr;

  for (;;) {   // ---- one piece: tiles [t0, t1) of unit (s, g)
    const int t0 = pos - unit0;
    const int t1 = T - t0 < end - pos ? T : t0 + (end - pos);
    const int tn = (n + kTile - 1) / kTile < t1 ? (n + kTile - 1) / kTile : t1;   // tiles that hold keys

    bf16x8 qop[NT][4];
    int rowpos[NT];
    RowState<NT> st;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = rb * kRows + 16 * nt + lr;
      const bool valid = r < p.R;
      const int j = valid ? r / p.G : 0;
      const int h = g * p.G + (valid ? r - j * p.G : 0);
      // selected entries lie below the length, and the one query at its end sees them all
      rowpos[nt] = valid && !gather ? L - p.nq + j : 0x7FFFFFFF;
      const uint16_t* qrow = p.q + (((int64_t)s * p.nq + j) * p.Hq + h) * kD + 32 * lg;
#pragma unroll
      for (int k = 0; k < 4; ++k) qop[nt][k] = as_bf16x8(valid ? load16(qrow + 8 * k) : u32x4{0u, 0u, 0u, 0u});
      st.m[nt] = -INFINITY;
      st.l[nt] = zero4();
      st.lx[nt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) st.o[nt][dt] = zero4();
    }
    const int minpos = gather ? 0x7FFFFFFF : L - p.nq + rb * kRows / p.G;         // position of the block's first row
    const int64_t head_row = (int64_t)s * p.kv.stride_seq + (int64_t)g * p.kv.stride_head;

    for (int c0 = t0; c0 < tn;) {   // ---- as many tiles as the table covers
      int c1 = tn;
      int page0 = 0, psub = 1;
      float inv_psub = 1.f;
      bool holes = false;            // some key that the table covers is absent
      if constexpr (ROWS == kQPages) {
        psub = p.kv.page_size >> 4;
        inv_psub = __builtin_amdgcn_rcpf((float)psub);
        const int64_t most = (int64_t)(kTab - 2) * psub / 2;
        if (c1 - c0 > most) c1 = c0 + (int)most;
        page0 = div_small(2 * c0, psub, inv_psub);
        const int last = (c1 * kTile < n ? c1 * kTile : n) - 1;
        const int np = div_small(last >> 4, psub, inv_psub) - page0 + 1;
        const int32_t* prow = p.kv.page_table + (int64_t)s * p.kv.max_pages_per_seq + page0;
        int bad = 0;
        for (int j = tid; j < np; j += kThreads) {
          const int pg = prow[j];
          const bool ok = (unsigned)pg < (unsigned)p.kv.num_pages;
          bad |= ok ? 0 : 1;
          sm.tab[j] = ok ? (uint32_t)((int64_t)pg * p.kv.stride_page + (int64_t)g * p.kv.stride_head) : kAbsent;
        }
        holes = __syncthreads_or(bad) != 0;
      } else if constexpr (ROWS == kQTable) {
        if (c1 - c0 > kTab / kTile) c1 = c0 + kTab / kTile;
        const int32_t* list = gather ? p.idx + ((int64_t)s * p.Hkv + g) * p.ld_idx : nullptr;
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
        }
        __syncthreads();
      }

      // row of a sub-tile's first key (uniform); `lim`: the last row of it that may be read (contiguous)
      auto sub_row = [&](int t, int& lim) -> int64_t {
        lim = 15;
        if constexpr (ROWS == kQContiguous) {
          if (t + 15 < n) return head_row + (int64_t)t * tok;
          lim = t < n ? n - 1 - t : 0;
          return head_row + (int64_t)(t < n ? t : n - 1) * tok;
        } else {
          if (t >= n) return 0;
          const int pi = div_small(t >> 4, psub, inv_psub);
          const uint32_t b = (uint32_t)__builtin_amdgcn_readfirstlane((int)sm.tab[pi - page0]);
          return b == kAbsent ? 0 : (int64_t)b + (int64_t)(t - pi * p.kv.page_size) * tok;
        }
      };
      // direct loads of tile c into ring slot `slot`
      auto issue = [&](int c, int slot) {
        const uint32_t dst = ring_lds + (uint32_t)(slot * TL::kBytes);
        if constexpr (ROWS == kQTable) {
          const uint32_t* tab = sm.tab + (c - c0) * kTile;
          auto row_at = [&](int r) { const uint32_t x = tab[r]; return x == kAbsent ? 0u : x; };
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < TL::kParts; ++e) {
              const uint32_t at = dst + 1024u * (uint32_t)(TL::kParts * h + e);
              const uint8_t* kp = p.kv.k + (uint64_t)row_at(16 * h + TL::k_row(lane, e)) * TL::kRow + 16 * TL::k_chunk(lane, e);
              const uint8_t* vp = p.kv.v + (uint64_t)row_at(16 * h + TL::v_row(lane, e)) * TL::kRow + 16 * TL::v_chunk(lane);
              dma16_hidden(reinterpret_cast<const uint16_t*>(kp), at);
              dma16_hidden(reinterpret_cast<const uint16_t*>(vp), at + TL::kV);
            }
          dma4_hidden(scales + (uint64_t)row_at(lane & 31) * kBlocks, dst + TL::kS);
        } else {
          int lim[2];
          const int64_t r0 = sub_row(c * kTile, lim[0]), r1 = sub_row(c * kTile + 16, lim[1]);
          const int64_t row[2] = {r0, r1};
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < TL::kParts; ++e) {
              const uint32_t at = dst + 1024u * (uint32_t)(TL::kParts * h + e);
              const int kr = TL::k_row(lane, e) < lim[h] ? TL::k_row(lane, e) : lim[h];
              const int vr = TL::v_row(lane, e) < lim[h] ? TL::v_row(lane, e) : lim[h];
              dma16_hidden(reinterpret_cast<const uint16_t*>(p.kv.k + row[h] * TL::kRow),
                           (uint32_t)kr * tok_bytes + 16u * (uint32_t)TL::k_chunk(lane, e), at);
              dma16_hidden(reinterpret_cast<const uint16_t*>(p.kv.v + row[h] * TL::kRow),
                           (uint32_t)vr * tok_bytes + 16u * (uint32_t)TL::v_chunk(lane), at + TL::kV);
            }
          const int hs = (lane >> 4) & 1;
          const int sr = lr < (hs ? lim[1] : lim[0]) ? lr : (hs ? lim[1] : lim[0]);
          dma4_hidden(scales + (uint64_t)((hs ? r1 : r0) + (int64_t)sr * tok) * kBlocks, dst + TL::kS);
        }
      };

      const int mine = c1 - c0 > wave ? (c1 - c0 - wave + kWaves - 1) / kWaves : 0;   // tiles of this wave
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // only tiles are counted from here on
      for (int i = 0; i < TL::kRing && i < mine; ++i) issue(c0 + wave + i * kWaves, i);
      for (int i = 0, slot = 0; i < mine; ++i, slot = slot + 1 == TL::kRing ? 0 : slot + 1) {
        const int c = c0 + wave + i * kWaves;
        const int later = mine - 1 - i < TL::kRing - 1 ? mine - 1 - i : TL::kRing - 1;
        wait_tiles<BITS>(later);
        TileRegs<BITS> tile;
        read_tile<BITS>(tile, sm.u.ring[wave][slot], lane);
        // key slot 4h + i of this lane: key c*32 + 16h + 4*lg + i
        const int key0 = c * kTile + 4 * lg;
        bool dirty = c * kTile + kTile > n || (!gather && c * kTile + kTile - 1 > minpos);
        uint32_t there = 0xFFu;
        if constexpr (ROWS == kQTable) {
          const uint64_t absent = __builtin_amdgcn_ballot_w64(sm.tab[(c - c0) * kTile + (lane & 31)] == kAbsent);
          dirty = dirty || (uint32_t)absent != 0u;
          const uint32_t ok = ~(uint32_t)absent >> (4 * lg);
          there = (ok & 0xFu) | ((ok >> 12) & 0xF0u);
        } else if (dirty || holes) {
          there = 0u;
#pragma unroll
          for (int i2 = 0; i2 < 8; ++i2) there |= key0 + 16 * (i2 >> 2) + (i2 & 3) < n ? 1u << i2 : 0u;
          if constexpr (ROWS == kQPages) {
            if (holes) {
              dirty = true;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int t = c * kTile + 16 * h;
                if (t < n && sm.tab[div_small(t >> 4, psub, inv_psub) - page0] == kAbsent) there &= h ? 0x0Fu : 0xF0u;
              }
            }
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read: it may be filled again
        if (i + TL::kRing < mine) issue(c + TL::kRing * kWaves, slot);
        tile_step<BITS, NT>(st, tile, qop, rowpos, p.scale_log2, dirty, there, key0, want_lx);
      }
      c0 = c1;
      if (ROWS != kQContiguous && c0 < tn) __syncthreads();   // the table is filled again
    }

    // ---- the four waves' states, through LDS
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float lx = st.lx[nt];
      lx += shfl_xor_f(lx, 16);
      lx += shfl_xor_f(lx, 32);
      const int r = 16 * nt + lr;
      if (lg == 0) {
        sm.u.merge.m[wave][r] = st.m[nt];
        sm.u.merge.l[wave][r] = st.l[nt][0];
        sm.u.merge.lx[wave][r] = lx;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float* dst = &sm.u.merge.o[wave][r][32 * lg + 8 * i];
        *reinterpret_cast<f32x4*>(dst) = f32x4{st.o[nt][0][i], st.o[nt][1][i], st.o[nt][2][i], st.o[nt][3][i]};
        *reinterpret_cast<f32x4*>(dst + 4) = f32x4{st.o[nt][4][i], st.o[nt][5][i], st.o[nt][6][i], st.o[nt][7][i]};
      }
    }
    __syncthreads();
    constexpr int kPer = kRows * kD / kThreads;            // outputs per thread: 8 or 16
    const int r = tid / (kD / kPer), d0 = (tid % (kD / kPer)) * kPer;
    float M = -INFINITY, Ls = 0.f, Lx = 0.f, acc[kPer];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm.u.merge.m[w][r]);
    const float Mu = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wt = exp2f(sm.u.merge.m[w][r] - Mu);
      Ls += wt * sm.u.merge.l[w][r];
      Lx += wt * sm.u.merge.lx[w][r];
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += wt * sm.u.merge.o[w][r][d0 + e];
    }

    const int row = rb * kRows + r;
    const bool row_valid = row < p.R;
    const int jrow = row_valid ? row / p.G : 0;
    const int64_t orow = ((int64_t)s * p.nq + jrow) * p.Hq + g * p.G + (row_valid ? row - jrow * p.G : 0);
    auto write_final = [&](float Mf, float Lf, float Lxf, const float (&a)[kPer]) {
      if (!row_valid) return;
      const float inv = Lf == 0.f ? 0.f : 1.f / Lf;        // no visible key: 0
      uint32_t w[kPer / 2];
#pragma unroll
      for (int e = 0; e < kPer; e += 2) w[e / 2] = pack_bf16x2(a[e] * inv, a[e + 1] * inv);
      uint16_t* dst = p.out + orow * kD + d0;
#pragma unroll
      for (int e = 0; e < kPer / 8; ++e)
        *reinterpret_cast<u32x4*>(dst + 8 * e) = u32x4{w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]};
      if (p.lse && d0 == 0) p.lse[orow] = Lxf == 0.f ? -INFINITY : (Mf + __log2f(Lxf)) * kLn2;
    };

    // ---- pieces of the unit: shares w0 .. w1
    const int w0 = unit0 / chunk, w1 = (unit0 + T - 1) / chunk;
    if (w0 == w1) {
      write_final(M, Ls, Lx, acc);
    } else {
      const __amdgpu_buffer_rsrc_t rec = make_rsrc(p.part, p.part_bytes);
      // a share leaves at most two records: of a unit that began before it, and of one that goes on after it
      auto at = [&](int w) { return (uint32_t)(2 * (w * p.n_rb + rb) + (w == w0 ? 1 : 0)) * (uint32_t)(kRec * 4); };
      auto store = [&](int w, float Mr, float Lr, float Lxr, const float (&a)[kPer]) {
        if (!row_valid) return;
        if (d0 == 0) store16_coherent(rec, at(w) + 16 * r, f32x4{Mr, Lr, Lxr, 0.f});
#pragma unroll
        for (int c = 0; c < kPer / 4; ++c)
          store16_coherent(rec, at(w) + 16 * kRows + 16 * (c * kThreads + tid),
                           f32x4{a[4 * c], a[4 * c + 1], a[4 * c + 2], a[4 * c + 3]});
      };
      float Mg, Lg, Lxg, ag[kPer];
      // records of shares first, first + step, ..., in that order, a batch of loads at a time
      auto merge = [&](int first, int count, int step) {
        Mg = -INFINITY;
        Lg = Lxg = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) ag[e] = 0.f;
        if (!row_valid) return;
        for (int k0 = 0; k0 < count; k0 += kGroup) {
          f32x4 sv[kGroup], ov[kGroup][kPer / 4];
#pragma unroll
          for (int u = 0; u < kGroup; ++u) {
            const bool ok = k0 + u < count;
            const uint32_t a = at(first + (k0 + u) * step);
            sv[u] = ok ? load16_coherent(rec, a + 16 * r) : f32x4{-INFINITY, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kPer / 4; ++c)
              ov[u][c] = ok ? load16_coherent(rec, a + 16 * kRows + 16 * (c * kThreads + tid)) : zero4();
          }
          float mb = Mg;
#pragma unroll
          for (int u = 0; u < kGroup; ++u) mb = fmaxf(mb, sv[u][0]);
          const float mbu = mb == -INFINITY ? 0.f : mb;
          const float sc = exp2f(Mg - mbu);
          Lg *= sc;
          Lxg *= sc;
#pragma unroll
          for (int e = 0; e < kPer; ++e) ag[e] *= sc;
#pragma unroll
          for (int u = 0; u < kGroup; ++u) {
            const float wt = exp2f(sv[u][0] - mbu);
            Lg += wt * sv[u][1];
            Lxg += wt * sv[u][2];
#pragma unroll
            for (int c = 0; c < kPer / 4; ++c)
#pragma unroll
              for (int i = 0; i < 4; ++i) ag[4 * c + i] += wt * ov[u][c][i];
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
      store(share, M, Ls, Lx, acc);
      // counter lines, each shares x row blocks: whole units, named by their first share; first groups, by the same;
      // other groups, by theirs, in which another unit's first group may begin
      const int region = !two ? 0 : grp == 0 ? 1 : 2;
      if (last_of((region * p.nW + g0) * p.n_rb + rb, gn)) {
        merge(g0, gn, 1);
        if (!two) {
          write_final(Mg, Lg, Lxg, ag);
        } else {
          __syncthreads();                                 // the group's first record is read: it is written again
          store(g0, Mg, Lg, Lxg, ag);
          if (last_of(w0 * p.n_rb + rb, (np + kGroup - 1) / kGroup)) {
            merge(w0, (np + kGroup - 1) / kGroup, kGroup);
            write_final(Mg, Lg, Lxg, ag);
          }
        }
      }
    }

    pos += t1 - t0;
    if (pos >= end) break;
    // the share goes on: the next unit from its first tile
    unit0 += T;
    if (++g == p.Hkv) {
      g = 0;
      ++s;
      n = unit_keys(p, s, L);
      T = unit_tiles(n);
    }
    __syncthreads();   // the merge buffer is read: the ring may be filled again
  }
}

template <int BITS, int NT>
hipError_t launch_rows(const QAttnParams& p, const QAttnPlan& pl, hipStream_t stream) {
  const dim3 grid((unsigned)pl.nblk), block(kThreads);
  if (pl.rows == kQContiguous) hipLaunchKernelGGL((qattn_kernel<BITS, NT, kQContiguous>), grid, block, 0, stream, p);
  else if (pl.rows == kQPages) hipLaunchKernelGGL((qattn_kernel<BITS, NT, kQPages>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((qattn_kernel<BITS, NT, kQTable>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace

QAttnPlan plan_qattn(int S, int Hkv, int Hq, int nq, int64_t entries, bool gather, bool paged, int page_size) {
  QAttnPlan pl{};
  const int64_t R = (int64_t)nq * (Hq / Hkv);
  pl.R = (int)(R < (1 << 30) ? R : (1 << 30));
  pl.nt = R <= 16 ? 1 : 2;
  pl.n_rb = (pl.R + 16 * pl.nt - 1) / (16 * pl.nt);
  // the kernel's page division is exact for 16-row sub-tiles numbered below 2^22
  pl.rows = gather ? kQTable : !paged ? kQContiguous : page_size % 16 == 0 && entries <= (1 << 26) - 64 ? kQPages : kQTable;
  pl.min_share = 8;
  const int64_t tiles = (int64_t)S * Hkv * (entries > 0 ? (entries + kTile - 1) / kTile : 1);
  int64_t nW = (tiles + pl.min_share - 1) / pl.min_share;
  const int64_t most = kMaxBlocks / pl.n_rb > 1 ? kMaxBlocks / pl.n_rb : 1;
  if (nW > most) nW = most;
  pl.nW = (int)nW;
  pl.nblk = tiles > INT32_MAX || entries > (1 << 30) || nW * pl.n_rb >= (1 << 22) ? -1 : nW * pl.n_rb;
  pl.counter_bytes = BD_WS_COUNTER_BYTES;
  const size_t rec = sizeof(float) * 16 * pl.nt * (4 + kD);
  pl.record_bytes = nW > 1 && pl.nblk > 0 ? align256(2 * rec * (size_t)pl.nblk) : 0;
  pl.ws_bytes = pl.counter_bytes + pl.record_bytes;
  return pl;
}

hipError_t launch_qattn(const QAttnParams& p, const QAttnPlan& pl, int bits, hipStream_t stream) {
  if (bits == 4) return pl.nt == 1 ? launch_rows<4, 1>(p, pl, stream) : launch_rows<4, 2>(p, pl, stream);
  return pl.nt == 1 ? launch_rows<8, 1>(p, pl, stream) : launch_rows<8, 2>(p, pl, stream);
}

}  // namespace bd
