// Building blocks of the attention kernels (gfx950): DMA of K, V, Q and dO tiles
// into swizzled LDS tiles, the two patterns that read MFMA operands from them,
// and the conversion and store of 32x32 MFMA results.
#pragma once

#include <type_traits>

#include "common.hpp"
#include "lds_dma.hpp"

namespace optimus {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazyRescale = 8.0f;  // forward: rescale when a query's maximum grows by more than 2^8
constexpr int kPrefetchMaxD = 80;     // head dims whose registers hold a tile's operands read ahead

// 2^x on the hardware exponential (v_exp_f32).  Every argument here is a
// logit minus a running maximum or the log-sum-exp.  Of a key that the query
// sees it is at most kLazyRescale (the maximum moves lazily) or, of the
// log-sum-exp, 0 up to rounding; results below the fp32 normal range flush to
// zero, which only drops weights under 2^-126.  Of a masked key it is -inf, or,
// in a causal backward, which masks the results, anything: later keys are not
// in the log-sum-exp, and the result may be +inf.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D>
struct Head {
  static constexpr int KS = D / 16;              // 16-wide contraction steps over d
  static constexpr int NF = (D + 31) / 32;       // 32-row fragments of a d-major result
};

// Pack eight fp32 (registers 8*half .. 8*half+7 of a 32x32 result) to bf16.
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t &v, int half) {
  u32x4_t r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = pack2(v[8 * half + 2 * e], v[8 * half + 2 * e + 1]);
  return as_bf16x8(r);
}

// Load this lane's token row (d values 16*kk + 8*hf .. +7 for each step kk)
// as B operands; zero for tokens >= S.
template <int D>
__device__ __forceinline__ void load_row_operand(bf16x8_t (&f)[Head<D>::KS], const bf16_t *src, bool valid,
                                                 int hf) {
#pragma unroll
  for (int kk = 0; kk < Head<D>::KS; ++kk)
    f[kk] = valid ? as_bf16x8(ldg16(src + kk * 16 + hf * 8)) : as_bf16x8(u32x4_t{0u, 0u, 0u, 0u});
}

// Store a d-major result through this wave's 8 KB LDS slot.  The lane of
// token t holds d values in 8-byte runs, so direct stores would touch 32 rows
// per instruction; here the runs go to LDS row t (256-byte rows, 16-byte
// chunk c stored at c ^ (t % 16)), and each lane then writes whole 16-byte
// row segments: a quarter-wave covers one row, four rows per instruction.
// First half: the runs of fragments 0 .. NF - 1, up to row D, into the slot.
template <int D, int NF>
__device__ __forceinline__ void dmajor_to_lds(const f32x16_t (&acc)[NF], float s, int lane, lds_char *slot) {
  const int t = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int nf = 0; nf < NF; ++nf) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d0 = nf * 32 + q * 8 + hf * 4;
      if (d0 < D) {
        const int c = d0 >> 3;
        *reinterpret_cast<__attribute__((address_space(3))) u32x2_t *>(slot + t * 256 + ((c ^ (t & 15)) << 4) +
                                                                        hf * 8) =
            u32x2_t{pack2(acc[nf][4 * q] * s, acc[nf][4 * q + 1] * s), pack2(acc[nf][4 * q + 2] * s, acc[nf][4 * q + 3] * s)};
      }
    }
  }
}

// Second half: rows of D from the slot.  dst is the row of the wave's first
// token, ld the row stride (elements), ntok the wave's tokens inside the
// sequence (the rest are not stored).
template <int D>
__device__ __forceinline__ void store_rows_lds(bf16_t *dst, size_t ld, int lane, const lds_char *slot, int ntok) {
  // LDS accesses of one wave run in order: the reads below see the writes
  const int j = lane & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = i * 4 + (lane >> 4);
    if (j * 8 < D && r < ntok) {
      const u32x4_t v =
          *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t *>(slot + r * 256 + ((j ^ (r & 15)) << 4));
      stg16(dst + r * ld + j * 8, v);
    }
  }
}

template <int D>
__device__ __forceinline__ void store_dmajor_lds(bf16_t *dst, size_t ld, const f32x16_t (&acc)[Head<D>::NF], float s,
                                                 int lane, lds_char *slot, int ntok) {
  dmajor_to_lds<D>(acc, s, lane, slot);
  store_rows_lds<D>(dst, ld, lane, slot, ntok);
}

constexpr int kDL = 128;  // LDS row length (elements)
constexpr int kMaxKT = 64;  // longest token tile of any kernel (bounds the DMA overhang past a tensor)

// Bytes of one tile of KT tokens (KT = 32: 8 KB; KT = 64: 16 KB).
template <int KT>
constexpr int tile_bytes() {
  return KT * kDL * 2;
}

__device__ __forceinline__ int tsw(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }
__device__ __forceinline__ int tile_off(int r, int c) { return r * (kDL * 2) + ((c ^ tsw(r)) << 4); }
__device__ __forceinline__ int perm23(int r) { return (r & ~0xC) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Per-lane byte offsets of this wave's DMA loads of one tile (KT/4 loads of
// 1 KB per tile, split over NW waves; tile-relative: the tile's first row and
// column go in the scalar offset).  perm stores token perm23(r) in row r.
template <int KT, int NW>
struct TileLoads {
  static constexpr int N = KT / 4 / NW;  // 1 KB loads per wave per tile
  static_assert(N >= 1 && N * NW * 4 == KT, "tile rows must split evenly over the waves");
};

template <int KT, int NW, int N>
__device__ __forceinline__ void tile_voff(uint32_t (&v)[N], int wid, int lane, int ld, bool perm) {
  static_assert(N == TileLoads<KT, NW>::N, "one offset per load");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int o = (wid * N + i) * 1024 + lane * 16;
    const int pr = o >> 8, c = ((o & 255) >> 4) ^ tsw(pr);
    v[i] = static_cast<uint32_t>(((perm ? perm23(pr) : pr) * ld + c * 8) * 2);
  }
}

// Issue one tile's DMA loads.  In the last tile of a sequence (rem < KT
// rows left) the rows past the sequence re-read the tile's first row: every
// product with those rows carries a zero weight, but a non-finite value in
// the next sequence would still turn that zero into NaN.
template <int KT, int NW, int N>
__device__ __forceinline__ void tile_issue(const u32x4_t &rsrc, uint32_t lds_tile, const uint32_t (&voff)[N],
                                           uint32_t soff, int wid, int lane, int rem, int ld, bool perm) {
  static_assert(N == TileLoads<KT, NW>::N, "one offset per load");
  const uint32_t sl = __builtin_amdgcn_readfirstlane(soff);
  if (rem >= KT) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      buffer_load_lds16(rsrc, __builtin_amdgcn_readfirstlane(lds_tile + (wid * N + i) * 1024), voff[i], sl);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int pr = (wid * N + i) * 4 + (lane >> 4);
      const int tok = perm ? perm23(pr) : pr;
      const uint32_t v = tok < rem ? voff[i] : voff[i] - static_cast<uint32_t>(tok * ld * 2);
      buffer_load_lds16(rsrc, __builtin_amdgcn_readfirstlane(lds_tile + (wid * N + i) * 1024), v, sl);
    }
  }
}

__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// This lane's LDS addresses of the two read patterns of a tile, relative to
// the tile.  They stay in registers, and the loops are unrolled over the two
// tile stages so that stage, fragment and step go in the reads' offset field:
// computed per read, the addresses were a sixth of the loops' vector work,
// which the matrix instructions of the SIMD's other waves compete with.
//
// row(f, kk): MFMA A operand (rows = tile rows 32f.., contraction = columns
// 16kk..) by ds_read_b128.
// col(nf, st): MFMA A operand (rows = columns 32nf.., contraction = tile rows
// 16st..) by two ds_read_b64_tr_b16.  With PERM, contraction index kk reads
// tile row 16st + perm23(kk): the operand then meets registers whose tokens
// come in the order a 32x32 MFMA result leaves them (bits 2 and 3 of the token
// index swapped), so one natural-order tile serves both the row reads and
// this read.  The transpose read takes each source lane's row address; lane
// half h (lanes 32h..) supplies rows 4h + (lane % 16) / 4 for elements 0..3
// and those rows + 8 for elements 4..7.
template <int D, bool PERM>
struct TileReads {
  using H = Head<D>;
  int row_off[H::KS], col_off[H::NF][2];
  // row_base, col_base: LDS offsets of the tiles the two patterns read, in stage 0
  __device__ __forceinline__ void init(int lane, int row_base, int col_base) {
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk) {
      row_off[kk] = row_base + tile_off(lane & 31, kk * 2 + (lane >> 5));
      asm volatile("" : "+v"(row_off[kk]));
    }
    const int k = (PERM ? 4 : 8) * (lane >> 5) + ((lane & 15) >> 2);
#pragma unroll
    for (int nf = 0; nf < H::NF; ++nf) {
      const int n = nf * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      col_off[nf][0] = col_base + tile_off(k, n >> 3) + (n & 7) * 2;
      col_off[nf][1] = col_base + tile_off(k + (PERM ? 8 : 4), n >> 3) + (n & 7) * 2;
      asm volatile("" : "+v"(col_off[nf][0]), "+v"(col_off[nf][1]));
    }
  }
  // stage: LDS address of the stage's offset 0
  __device__ __forceinline__ bf16x8_t row(const lds_char *stage, int f, int kk) const {
    return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8_t *>(stage + f * 32 * kDL * 2 + row_off[kk]);
  }
  __device__ __forceinline__ bf16x8_t col(const lds_char *stage, int nf, int st) const {
    const lds_char *q = stage + st * 16 * kDL * 2;
    return lds_read_tr(q + col_off[nf][0], q + col_off[nf][1]);
  }
};

// A operands of a token-contracting product (columns nf*32.. of a tile,
// contraction over its rows), read ahead of the work they wait on when the
// head is small enough for the registers (PRE); otherwise read at use.
template <int D, int KT, bool PRE, bool PERM>
struct ColOperands {
  bf16x8_t v[PRE ? KT / 16 : 1][PRE ? Head<D>::NF : 1];
  __device__ __forceinline__ void fetch(const lds_char *stage, const TileReads<D, PERM> &r) {
    if constexpr (PRE) {
#pragma unroll
      for (int st = 0; st < KT / 16; ++st)
#pragma unroll
        for (int nf = 0; nf < Head<D>::NF; ++nf) v[st][nf] = r.col(stage, nf, st);
    }
  }
  __device__ __forceinline__ bf16x8_t get(const lds_char *stage, const TileReads<D, PERM> &r, int nf, int st) const {
    if constexpr (PRE)
      return v[st][nf];
    else
      return r.col(stage, nf, st);
  }
};

template <int N>
using Stage = std::integral_constant<int, N>;

}  // namespace optimus
