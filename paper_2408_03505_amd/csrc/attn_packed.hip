// Attention within the sequences of a packed batch, forward and backward.
//
// Layout: qkv is [tokens, (heads + 2 kv_heads) * D] with columns
// [heads + 2 kv_heads][D]: queries, keys, values; query head h reads key head
// h / (heads / kv_heads).  o, dO are [tokens, heads * D]; lse and the
// backward's D vector are [heads, tokens] fp32.  The sequences lie end to end;
// a work list (packed_plan.hip) names a sequence and kPackedRows of its tokens
// for each workgroup and head, the longest sequences first.  Rows of no
// sequence are neither read nor written.
//
// The mathematics and the products' orientation are those of the dense
// attention kernels (S^T = K Q^T, O^T += V^T P^T, online softmax with a lazily
// moved maximum; the backward recomputes P from lse).  What differs:
//  - A sequence's tiles of one head are loaded through one buffer resource, which
//    begins at its first row (a 64-bit address) and ends with its last: rows past
//    it read as zero, and a non-finite value behind a sequence never reaches it.
//    Lanes whose LDS columns lie past the head's width ask for nothing.
//  - With `causal`, a query's keys end with itself: key tiles past a
//    workgroup's last query (query tiles before its first key, in dK/dV) are
//    skipped, and those on the diagonal are masked element by element.
//  - dK/dV runs over the queries of every head that shares the key head, in
//    head order, so the gradients of shared heads are summed in the
//    accumulators, with no atomics and always in the same order.
//
// What bounds it: the matrix cores under the card's power limit on long sequences
// (16 heads of 128 over 7936 + 515 + 1 tokens: busy 0.58 of the time at 1.8 GHz in
// the forward, 0.66 at 1.7 in dQ, 0.62 at 1.8 in dK/dV), with as many LDS bytes
// as the LDS can deliver beside them (each 32x32x16 product reads 1 KB, which takes
// the CU as long as its four SIMDs take to use it).  On short and ragged ones (40
// images of 68 to 1020 tokens, 16 heads of 80, at 2.0 GHz) the matrix cores are busy
// 0.33 to 0.36 of the time and the vector units 0.53 (forward), 0.42 (dQ) and 0.35.
// In the forward that is most of it: a wave's tile takes 320 cycles of products, but
// 16 exponentials and 120 other vector instructions, which take a SIMD 520 (10 and 3
// each in loops of their own), and the two overlap little.  The rest waits: a
// workgroup has 18 tiles on average, before which nothing hides its work item, its
// queries and its first tiles (waves past a sequence's end idle for 6% of the tiles).
// Below some 200 tokens each kernel is bound by its bytes (112 x 128 tokens, 16 heads
// of 80: forward 31 us for 147 MB, backward 97 for 441).  Figures beside the kernels
// are medians of a kernel trace; rates count 4, 6 and 8 flops per query, key and element of a head in the
// forward, dQ (S, dP and dQ) and dK/dV (S, dP, dV and dK).
#include <float.h>
#include <math.h>

#include <algorithm>

#include "attn_tiles.hpp"
#include "common.hpp"
#include "kernels.hpp"
#include "lds_dma.hpp"

namespace optimus {

namespace {

// Work item and head of this workgroup.  Workgroup i runs on XCD i % 8: with
// a multiple of 8 heads each XCD takes one eighth of them, so the tiles of one
// sequence and head, and of heads that share keys, share the XCD's L2.  Items
// go longest first on every XCD.
__device__ __forceinline__ void packed_item(int heads, int &item, int &h) {
  const int pid = blockIdx.x;
  if (heads % 8 == 0) {
    const int per = heads / 8, local = pid >> 3;
    item = local / per;
    h = (pid & 7) * per + local % per;
  } else {
    item = pid / heads;
    h = pid % heads;
  }
}

// The item's sequence and first row in it, kept inside the tensors whatever
// the list holds; false for the empty items behind the list's end.
__device__ __forceinline__ bool load_item(const PackedPlan *plan, int tokens, int i, int &first, int &len, int &row) {
  const PackedItem it = plan->item[i];
  first = __builtin_amdgcn_readfirstlane(min(max(it.first, 0), tokens));
  len = __builtin_amdgcn_readfirstlane(min(max(it.len, 0), tokens - first));
  row = __builtin_amdgcn_readfirstlane(max(it.row, 0));
  return row < len;
}

// What a workgroup of the forward and of dQ does: its sequence, each wave's head
// and first query, and the keys that some query of it sees.  Four waves take an
// item's 128 queries of one head; or, where a multiple of four heads share their
// keys, 32 queries of four heads.  Then the waves see the same keys with `causal`
// too, and fewer waves lie past a sequence's end (24 prompts of 30 to 1625
// tokens, 32 heads on 8, causal: forward 126 -> 116 us, dQ 195 -> 184).
struct QueryWork {
  int first, len;     // the sequence
  int h, kvh, q0;     // the wave's head, its key head and its first query
  int keys;           // the workgroup's keys
  int wave_keys;      // those that some query of the wave sees; 0: no queries
  int all_see;        // those that all of them see
};

__device__ __forceinline__ bool query_work(const PackedAttnArgs &p, int wid, QueryWork &w) {
  int item, row;
  const bool shared = p.shared4;
  packed_item(shared ? p.heads / 4 : p.heads, item, w.h);
  if (!load_item(p.plan, p.tokens, shared ? item >> 2 : item, w.first, w.len, row)) return false;
  if (shared) {
    row += 32 * (3 - (item & 3));
    if (row >= w.len) return false;
    w.h = w.h * 4 + wid;
    w.q0 = row;
    w.keys = p.causal ? min(w.len, row + 32) : w.len;
  } else {
    w.q0 = row + wid * 32;
    w.keys = p.causal ? min(w.len, row + kPackedRows) : w.len;
  }
  w.kvh = w.h / (p.heads / p.kv_heads);
  w.wave_keys = w.q0 >= w.len ? 0 : p.causal ? min(w.len, w.q0 + 32) : w.len;
  w.all_see = p.causal ? min(w.len, w.q0 + 1) : w.len;
  return true;
}

// Per-lane byte offsets of this wave's loads of a tile (rows ld elements
// apart); lanes past the head's width ask for nothing (a sequence may span 4 GiB).
template <int D, int KT, int NW, int N>
__device__ __forceinline__ void packed_voff(uint32_t (&v)[N], int wid, int lane, int ld, bool perm) {
  static_assert(N == TileLoads<KT, NW>::N, "one offset per load");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int o = (wid * N + i) * 1024 + lane * 16;
    const int pr = o >> 8, c = ((o & 255) >> 4) ^ tsw(pr);
    v[i] = c * 8 < D ? static_cast<uint32_t>(((perm ? perm23(pr) : pr) * ld + c * 8) * 2) : kPastEnd;
  }
}

// One tensor's tiles of one sequence and head, loaded in order: a buffer
// resource from the head's first column in the first row on, which ends with
// the sequence's last row, and the next tile's byte offset in it.  A load is
// then one addition and two instructions per kilobyte: set up anew for each
// tile, the loads' scalar instructions held each wave up by a tenth of its time.
template <int D, int KT, int NW>
struct PackedLoads {
  static constexpr int NL = TileLoads<KT, NW>::N;
  u32x4_t rsrc;
  uint32_t voff[NL], soff, step, wbase;
  __device__ __forceinline__ void init(const bf16_t *src, int rows, int ld, uint32_t lds_base, int wid, int lane,
                                       bool perm) {
    packed_voff<D, KT, NW>(voff, wid, lane, ld, perm);
    step = static_cast<uint32_t>(KT) * ld * 2;
    wbase = __builtin_amdgcn_readfirstlane(lds_base + wid * NL * 1024);
    start(src, rows, ld);
  }
  // the next tile is the one at src, of `rows` rows to the sequence's end
  __device__ __forceinline__ void start(const bf16_t *src, int rows, int ld) {
    rsrc = make_rsrc(src, (static_cast<uint32_t>(rows - 1) * ld + D) * 2);
    soff = 0;
  }
  // into the tile OFF bytes on in LDS
  template <int OFF>
  __device__ __forceinline__ void issue() {
    issue_each<OFF, 0>();
    soff += step;
  }
  template <int OFF, int I>
  __device__ __forceinline__ void issue_each() const {
    if constexpr (I < NL) {
      issue_lds16<OFF + I * 1024>(rsrc, wbase, voff[I], soff);
      issue_each<OFF, I + 1>();
    }
  }
};

// LDS address of this lane's first transposed read of a tile's columns D - 16 ..
// D - 1 as the operand of a 16x16x32 product: lanes 16 g .. 16 g + 15 read the eight
// tokens that 16-lane groups of a packed result hold (Result::add), 4 (g / 2) + 16
// (g % 2) and those 8 further on (second_read's).
template <int D, bool PERM>
__device__ __forceinline__ int tail_first(int lane, uint32_t lds0) {
  const int g = lane >> 4, k = 16 * (g & 1) + (PERM ? 4 : 8) * (g >> 1) + ((lane & 15) >> 2);
  const int n = D - 16 + 4 * (lane & 3);
  return lds0 + tile_off(k, n >> 3) + (n & 7) * 2;
}
// 8 rows further with PERM, else 4 (the swizzle differs in one bit)
template <bool PERM>
__device__ __forceinline__ int second_read(int c) {
  return PERM ? (c ^ 32) + 8 * kDL * 2 : (c ^ 16) + 4 * kDL * 2;
}

// TileReads with every address a whole LDS address, so that stage, tile,
// fragment and step all go in the reads' offset field.
template <int D, bool PERM>
struct PackedReadsR {
  TileReads<D, PERM> t;
  int tail_off[2];
  __device__ __forceinline__ void init(int lane, uint32_t lds0) {
    t.init(lane, lds0, lds0);
    tail_off[0] = tail_first<D, PERM>(lane, lds0);
    tail_off[1] = second_read<PERM>(tail_off[0]);
  }
  __device__ __forceinline__ bf16x8_t tail(int base) const {
    return lds_read_tr(reinterpret_cast<const lds_char *>(static_cast<uint32_t>(tail_off[0] + base)),
                       reinterpret_cast<const lds_char *>(static_cast<uint32_t>(tail_off[1] + base)));
  }
  __device__ __forceinline__ bf16x8_t row(int base, int f, int kk) const {
    return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8_t *>(
        static_cast<uint32_t>(t.row_off[kk] + base + f * 32 * kDL * 2));
  }
  __device__ __forceinline__ bf16x8_t col(int base, int nf, int st) const {
    const int o = base + st * 16 * kDL * 2;
    return lds_read_tr(reinterpret_cast<const lds_char *>(static_cast<uint32_t>(t.col_off[nf][0] + o)),
                       reinterpret_cast<const lds_char *>(static_cast<uint32_t>(t.col_off[nf][1] + o)));
  }
};

// The same, and reads of fp32 vectors in the order of a result's registers,
// from few registers.  The tile swizzle is an XOR of the 16-byte chunk, so steps
// along the columns are an XOR of the first one's address: one vector
// instruction per read, where registers are what limits the kernel.
template <int D, bool PERM>
struct PackedReads {
  int row0, col0, vec0, tail0;
  __device__ __forceinline__ void init(int lane, uint32_t lds0) {
    row0 = lds0 + tile_off(lane & 31, lane >> 5);
    const int k = (PERM ? 4 : 8) * (lane >> 5) + ((lane & 15) >> 2);
    const int n = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    col0 = lds0 + tile_off(k, n >> 3) + (n & 7) * 2;
    vec0 = lds0 + (lane >> 5) * 16;
    tail0 = tail_first<D, PERM>(lane, lds0);
    asm volatile("" : "+v"(row0), "+v"(col0), "+v"(vec0));
  }
  // Called in the loop: keeps its addresses from being computed, and held in
  // registers, outside it.
  __device__ __forceinline__ void local() { asm volatile("" : "+v"(row0), "+v"(col0)); }
  template <class T>
  __device__ static __forceinline__ T at(uint32_t addr) {
    return *reinterpret_cast<const __attribute__((address_space(3))) T *>(addr);
  }
  __device__ __forceinline__ bf16x8_t row(int base, int f, int kk) const {
    return at<bf16x8_t>((row0 ^ (kk << 5)) + base + f * 32 * kDL * 2);
  }
  __device__ __forceinline__ bf16x8_t col(int base, int nf, int st) const {
    const int o = base + st * 16 * kDL * 2, c = col0 ^ (nf << 6);
    return lds_read_tr(reinterpret_cast<const lds_char *>(c + o),
                       reinterpret_cast<const lds_char *>(second_read<PERM>(c) + o));
  }
  __device__ __forceinline__ bf16x8_t tail(int base) const {
    return lds_read_tr(reinterpret_cast<const lds_char *>(tail0 + base),
                       reinterpret_cast<const lds_char *>(second_read<PERM>(tail0) + base));
  }
  __device__ __forceinline__ f32x4_t vec(int base) const { return at<f32x4_t>(vec0 + base); }
};

// A value of each lane's token (lane % 32) for results that hold tokens 0..15 (lo)
// and 16..31 (hi) in every 16 lanes.
__device__ __forceinline__ void by_halves(uint32_t a, uint32_t b, uint32_t &lo, uint32_t &hi) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  lo = r[0];
  hi = r[1];
}
__device__ __forceinline__ void by_halves(float v, float &lo, float &hi) {
  uint32_t a, b;
  by_halves(__float_as_uint(v), __float_as_uint(v), a, b);
  lo = __uint_as_float(a);
  hi = __uint_as_float(b);
}

// The sum of tiles' products with a 32x32 result, [D][32 tokens]: fragments of 32
// rows, and for a head that ends with 16 more (80) two of 16 by 16 tokens, where a
// third 32-row fragment would spend twice the matrix and LDS time on them (8192
// tokens, 16 heads of 80: forward 374 -> 366 us, backward 1136 -> 1099).
template <int D>
struct Result {
  static constexpr int NF = D / 32;
  static constexpr bool TAIL = D % 32 != 0;
  static_assert(!TAIL || D % 32 == 16, "a half fragment at the end");
  static constexpr int MFMAS = 2 * NF + 2 * TAIL, READS = 4 * NF + 2 * TAIL;  // of add
  f32x16_t w[NF];
  f32x4_t t[2];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < NF; ++i) w[i] = f32x16_t{};
    t[0] = t[1] = f32x4_t{};
  }
  // each token's column by the value of its lanes
  __device__ __forceinline__ void scale(float s) {
#pragma unroll
    for (int i = 0; i < NF; ++i) w[i] *= s;
    if constexpr (TAIL) {
      float lo, hi;
      by_halves(s, lo, hi);
      t[0] *= lo;
      t[1] *= hi;
    }
  }
  // += X^T s, s a 32x32 result [token of the tile][token], X the tile at base.
  // s (P, or dS) is rounded to bf16 here: the other operand is bf16, and matrix
  // instructions that take fp32 run at a sixteenth of the rate.  A weight is off by up
  // to 2^-8 of itself, and the sums of the forward (l, and the lse) are of the unrounded
  // ones; o is off by 1.9 to 2.0e-3 (2-norm, relative) where rounding o alone gives 1.5
  // to 1.6e-3, with the gradients by 2.0 to 2.4e-3 where it gives 1.4 to 1.7e-3.
  template <class Reads>
  __device__ __forceinline__ void add(const Reads &rd, int base, const f32x16_t &s) {
    bf16x8_t b[2];
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      b[st] = pack8(s, st);
#pragma unroll
      for (int i = 0; i < NF; ++i) w[i] = mfma32(rd.col(base, i, st), b[st], w[i]);
    }
    if constexpr (TAIL) {
      // Lanes 16 r .. 16 r + 15 of b[st] hold tokens 16 (r % 2) .. + 15 and, of the
      // tile, 4 (r / 2) + 16 st ..; the product takes all of one half's tokens.
      const u32x4_t x = __builtin_bit_cast(u32x4_t, b[0]), y = __builtin_bit_cast(u32x4_t, b[1]);
      u32x4_t lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t l, h;
        by_halves(x[e], y[e], l, h);
        lo[e] = l;
        hi[e] = h;
      }
      const bf16x8_t v = rd.tail(base);
      t[0] = mfma16(v, as_bf16x8(lo), t[0]);
      t[1] = mfma16(v, as_bf16x8(hi), t[1]);
    }
  }
  // times s, through the wave's LDS slot, to rows dst, dst + ld ..
  __device__ __forceinline__ void store(bf16_t *dst, size_t ld, float s, int lane, lds_char *slot, int ntok) const {
    dmajor_to_lds<D>(w, s, lane, slot);
    if constexpr (TAIL) {
      float lo, hi;
      by_halves(s, lo, hi);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int tok = 16 * i + (lane & 15), c = D / 8 - 2 + (lane >> 5);
        const float f = i ? hi : lo;
        *reinterpret_cast<__attribute__((address_space(3))) u32x2_t *>(slot + tok * 256 + ((c ^ (tok & 15)) << 4) +
                                                                        ((lane >> 4) & 1) * 8) =
            u32x2_t{pack2(t[i][0] * f, t[i][1] * f), pack2(t[i][2] * f, t[i][3] * f)};
      }
    }
    store_rows_lds<D>(dst, ld, lane, slot, ntok);
  }
};

// ------------------------------------------------------------------ forward
//
// Each wave runs one tile ahead of itself: the products S(t + 1) = K Q^T are in
// one straight piece of code with the exponentials of tile t, and the running
// maximum of tile t + 1 with the products O += P V of tile t, so that vector
// instructions fill the time that a matrix instruction leaves the SIMD's issue
// free.  (Left to different waves they hardly overlap: with S, softmax and PV in
// turn and three waves per SIMD, the matrix cores were busy 0.45 of the time and
// the vector units 0.45.)  Tile t + 2's keys and tile t + 1's values are loaded
// meanwhile.
//
// 16 heads of 128 over 7936 + 515 + 1 tokens 484 us (1070 TFLOP/s); 16 of 80 over
// the 40 images 71 (660); 32 of 128 on 8, causal, 24 prompts of 30 to 1625 tokens
// 143 (690; 118 to 130 in a loop of this kernel alone).  A tile's loads, LDS reads and
// exponentials, each left out of a copy, took 18, 61 and 13 us of 523 at 8192
// tokens: none alone is what it waits for.

// The next N instructions of a kind in the order wanted of the scheduler.
constexpr int kSchedVector = 0x2, kSchedMfma = 0x8, kSchedLds = 0x100, kSchedTrans = 0x400;
template <int KIND, int N>
__device__ __forceinline__ void sched_group() {
  __builtin_amdgcn_sched_group_barrier(KIND, N, 0);
}

__device__ __forceinline__ float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float max16(const f32x16_t &s) {
  float a = fmaxf(s[0], s[1]), b = fmaxf(s[8], s[9]);
#pragma unroll
  for (int i = 2; i < 8; ++i) a = fmaxf(a, s[i]), b = fmaxf(b, s[i + 8]);
  return fmaxf(a, b);
}

template <int D, int WPE>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(WPE, WPE))) void
packed_fwd_kernel(PackedAttnArgs p) {
  using H = Head<D>;
  constexpr int KT = 32, TB = tile_bytes<KT>(), VB = 2 * TB;  // K, K, V, V
  using Loads = PackedLoads<D, KT, 4>;
  constexpr int NL = Loads::NL;
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_char *)smem_raw));

  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  QueryWork w;
  if (!query_work(p, wid, w)) return;
  const int first = w.first, len = w.len, h = w.h, kvh = w.kvh, q0 = w.q0;
  const int A = p.heads * D, ld = A + 2 * p.kv_heads * D;
  const int q = q0 + (lane & 31);
  const bf16_t *seq = p.qkv + static_cast<size_t>(first) * ld;
  const bf16_t *kp = seq + A + kvh * D, *vp = kp + p.kv_heads * D;

  Loads lk, lv;
  lk.init(kp, len, ld, lds0, wid, lane, false);
  lv.init(vp, len, ld, lds0 + VB, wid, lane, true);

  bf16x8_t qf[H::KS];
  load_row_operand<D>(qf, seq + static_cast<size_t>(q) * ld + h * D, q < len, hf);

  Result<D> acc;
  acc.zero();
  // m starts below every scaled logit but finite: a logit of -inf then weighs
  // exp2(-inf - m) = 0 also where the tiles so far hold no other (from m = -inf it
  // would weigh NaN)
  float m = -FLT_MAX, top = -INFINITY, l = 0.f;
  const float c = kLog2e / sqrtf(static_cast<float>(D));

  PackedReadsR<D, false> rd;
  rd.init(lane, lds0);
  // key tiles of the workgroup and of the wave; the first tile that some query
  // of the wave does not see whole, and the keys of this lane's query
  const int nk = (w.keys + KT - 1) / KT, nkw = (w.wave_keys + KT - 1) / KT;
  const int tmask = w.all_see / KT;
  const int lim = p.causal ? min(len, q + 1) : len;

  auto logits = [&](int base, f32x16_t &s) {
    s = f32x16_t{};
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk) s = mfma32(rd.row(base, 0, kk), qf[kk], s);
  };
  auto mask = [&](int t, f32x16_t &s) {
    const int left = lim - t * KT - hf * 4;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if ((i >> 2) * 8 + (i & 3) >= left) s[i] = -INFINITY;
  };
  // Raw logits are scaled by c > 0, so the scaled maximum is c times the raw
  // one.  The reference maximum m of a query moves only when a logit exceeds it
  // by more than kLazyRescale (log2 units; `top` is that in raw logits): O = acc / l
  // and lse = m + log2 l hold for any m.  ms is the maximum over the half of the
  // tile's keys that this lane holds, which is enough to see whether any moves.
  // (It moves at the first logit above -inf: those lie above -FLT_MAX, which c < 1
  // takes far above m's start; `top` stays -inf until then, as m's start / c does.)
  auto move_max = [&](float ms) {
    if (__any(ms > top)) {
      const float mt = max_halves(ms) * c;
      const float mn = mt > m + kLazyRescale ? mt : m;
      const float alpha = exp2_hw(m - mn);  // 0 at the first move, 1 where m stays
      m = mn;
      top = (mn + kLazyRescale) / c;
      l *= alpha;
      acc.scale(alpha);
    }
  };

  f32x16_t s0, s1;
  lk.template issue<0>();
  lv.template issue<0>();
  if (nk > 1) {
    lk.template issue<TB>();
    wait_vmcnt<2 * NL>();
  } else {
    wait_vmcnt<NL>();
  }
  block_barrier();
  if (nkw > 0) {
    logits(0, s0);
    if (tmask <= 0) mask(0, s0);
    move_max(max16(s0));
  }
  auto tile = [&](auto stage, f32x16_t &s, f32x16_t &next, int t) {
    constexpr int ST = stage.value;
    wait_vmcnt<0>();  // this wave's loads of V(t) and K(t + 1) have landed
    // every wave's have, and every wave is done with K(t) and V(t - 1), whose
    // buffers the next loads refill
    block_barrier();
    if (t + 2 < nk) lk.template issue<ST * TB>();
    if (t + 1 < nk) lv.template issue<(1 - ST) * TB>();
    if (t >= nkw) return;  // waves that see none of the tile's keys only load and synchronise
    // A wave's products go before the other waves' loads and prologues: from S(t + 1)
    // on, 16 heads of 128 over 8192 tokens 553 -> 535 us, of 64 295 -> 287, but of 80,
    // with three workgroups to a CU, 368 -> 385; there from P V on, 361.
    constexpr bool kFromLogits = D != 80;
    if constexpr (kFromLogits) __builtin_amdgcn_s_setprio(1);
    // (past the wave's last tile the logits are of stale data and not used)
    logits((1 - ST) * TB, next);
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      s[i] = exp2_hw(__builtin_fmaf(s[i], c, -m));
      s[i + 1] = exp2_hw(__builtin_fmaf(s[i + 1], c, -m));
      l0 += s[i];
      l1 += s[i + 1];
    }
    l += l0 + l1;
    if constexpr (!kFromLogits) __builtin_amdgcn_s_setprio(1);
    acc.add(rd, VB + ST * TB, s);
    __builtin_amdgcn_s_setprio(0);
    float ms = max16(next);
    // The order wanted: the keys' operands, under whose latency the first
    // exponentials run, then S(t + 1) with the other exponentials and the values'
    // operands between its products, then P V with the maximum.
    sched_group<kSchedLds, H::KS>();
    sched_group<kSchedVector, 20>();
    sched_group<kSchedTrans, 8>();
#pragma unroll
    for (int i = 0; i < H::KS; ++i) {
      sched_group<kSchedMfma, 1>();
      sched_group<kSchedVector, 20 / H::KS>();
      sched_group<kSchedTrans, (8 + H::KS - 1) / H::KS>();
      sched_group<kSchedLds, (Result<D>::READS + H::KS - 1) / H::KS>();
    }
#pragma unroll
    for (int i = 0; i < Result<D>::MFMAS; ++i) {
      sched_group<kSchedMfma, 1>();
      sched_group<kSchedVector, 2>();
    }
    if (t + 1 < nkw) {
      if (t + 1 >= tmask) {
        mask(t + 1, next);
        ms = max16(next);
      }
      move_max(ms);
    }
  };
  for (int t = 0; t < nk; t += 2) {
    tile(Stage<0>(), s0, s1, t);
    if (t + 1 < nk) tile(Stage<1>(), s1, s0, t + 1);
  }
  block_barrier();  // every wave is done with the tile buffers, which the output slots reuse

  const float lt = l + __shfl_xor(l, 32, kWave);
  if (q < len && hf == 0) p.lse[static_cast<size_t>(h) * p.tokens + first + q] = (m + log2f(lt)) / kLog2e;
  acc.store(p.o + static_cast<size_t>(first + q0) * A + h * D, A, 1.0f / lt, lane, (lds_char *)smem_raw + wid * 8192,
            len - q0);
}

// ------------------------------------------------------------------ backward: dQ and D
//
// As in the forward a wave runs ahead of itself, here within a tile: dP(t) =
// V dO^T is in one piece of code with the exponentials of tile t, S(t + 1) with
// dS(t) = P (dP - D), and dQ^T += K^T dS^T follows.  Three stages of K (tile t
// for dQ, t + 1 for S, t + 2 in flight) and two of V.
//
// The three sets as for the forward: 665 us (1170 TFLOP/s), 99 (710), 203 (720).
// It also leaves -lse sqrt(D) and -D_i for the dK/dV kernel.

template <int D, int WPE>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(WPE, WPE))) void
packed_bwd_dq_kernel(PackedAttnArgs p) {
  using H = Head<D>;
  constexpr int KT = 32, TB = tile_bytes<KT>(), VB = 3 * TB;  // K, K, K, V, V
  using Loads = PackedLoads<D, KT, 4>;
  constexpr int NL = Loads::NL;
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_char *)smem_raw));

  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  QueryWork w;
  if (!query_work(p, wid, w)) return;
  const int first = w.first, len = w.len, h = w.h, kvh = w.kvh, q0 = w.q0;
  const int A = p.heads * D, ld = A + 2 * p.kv_heads * D;
  const int q = q0 + (lane & 31);
  const bool qvalid = q < len;
  const bf16_t *seq = p.qkv + static_cast<size_t>(first) * ld;
  const bf16_t *kp = seq + A + kvh * D, *vp = kp + p.kv_heads * D;
  const size_t orow = static_cast<size_t>(first + q) * A + h * D;
  const size_t vec = static_cast<size_t>(h) * p.tokens + first + q;

  Loads lk, lv;
  lk.init(kp, len, ld, lds0, wid, lane, false);
  lv.init(vp, len, ld, lds0 + VB, wid, lane, false);

  bf16x8_t qf[H::KS], df[H::KS];
  load_row_operand<D>(qf, seq + static_cast<size_t>(q) * ld + h * D, qvalid, hf);
  load_row_operand<D>(df, p.dO + orow, qvalid, hf);
  float dd = 0.f;  // D_i (this lane holds half of the d values of its query)
  if (qvalid) {
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk) {
      const u32x4_t ow = ldg16(p.o + orow + kk * 16 + hf * 8);
      const u32x4_t dw = __builtin_bit_cast(u32x4_t, df[kk]);
#pragma unroll
      for (int e = 0; e < 4; ++e) dd += lo_bf(ow[e]) * lo_bf(dw[e]) + hi_bf(ow[e]) * hi_bf(dw[e]);
    }
  }
  dd += __shfl_xor(dd, 32, kWave);
  const float c = kLog2e / sqrtf(static_cast<float>(D));
  const float lse2 = qvalid ? p.lse[vec] * kLog2e : 0.f;
  if (qvalid && hf == 0) {
    p.nlse[vec] = -p.lse[vec] * sqrtf(static_cast<float>(D));
    p.ndvec[vec] = -dd;
  }

  Result<D> acc;
  acc.zero();
  const int nk = (w.keys + KT - 1) / KT, nkw = (w.wave_keys + KT - 1) / KT;
  const int tmask = w.all_see / KT;
  const int lim = p.causal ? min(len, q + 1) : len;
  // K: row reads for S^T and the permuted column reads; V: row reads
  PackedReadsR<D, true> rd;
  rd.init(lane, lds0);
  auto logits = [&](int base, f32x16_t &s) {
    s = f32x16_t{};
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk) s = mfma32(rd.row(base, 0, kk), qf[kk], s);
  };

  // loads in the order K(0), V(0), K(1), then V(t + 1), K(t + 2) in tile t
  f32x16_t s0, s1;
  lk.template issue<0>();
  lv.template issue<0>();
  if (nk > 1) {
    lk.template issue<TB>();
    wait_vmcnt<2 * NL>();
  } else {
    wait_vmcnt<NL>();
  }
  block_barrier();
  if (nkw > 0) logits(0, s0);
  auto tile = [&](auto kstage, auto vstage, f32x16_t &s, f32x16_t &next, int t) {
    constexpr int KS0 = kstage.value * TB, KS1 = (kstage.value + 1) % 3 * TB, KS2 = (kstage.value + 2) % 3 * TB;
    constexpr int VS = VB + vstage.value * TB;
    wait_vmcnt<0>();  // this wave's loads of V(t) and K(t + 1)
    // everyone's have landed, and everyone is done with K(t - 1) and V(t - 1)
    block_barrier();
    if (t + 1 < nk) lv.template issue<(1 - vstage.value) * TB>();
    if (t + 2 < nk) lk.template issue<KS2>();
    if (t >= nkw) return;  // waves that see none of the tile's keys only load and synchronise
    f32x16_t dp{};
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk) dp = mfma32(rd.row(VS, 0, kk), df[kk], dp);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = exp2_hw(__builtin_fmaf(s[i], c, -lse2));
    // (past the wave's last tile the logits are of stale data and not used)
    logits(KS1, next);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= dp[i] - dd;  // dS^T
    sched_group<kSchedLds, H::KS>();
    sched_group<kSchedVector, 8>();
    sched_group<kSchedTrans, 4>();
#pragma unroll
    for (int i = 0; i < H::KS; ++i) {
      sched_group<kSchedMfma, 1>();
      sched_group<kSchedVector, 8 / H::KS>();
      sched_group<kSchedTrans, (12 + H::KS - 1) / H::KS>();
      sched_group<kSchedLds, 1>();
    }
#pragma unroll
    for (int i = 0; i < H::KS; ++i) {
      sched_group<kSchedMfma, 1>();
      sched_group<kSchedVector, (32 + H::KS - 1) / H::KS>();
    }
    if (t >= tmask) {
      // register i is key t*KT + 8(i/4) + 4 hf + i%4
      const int left = lim - t * KT - hf * 4;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if ((i >> 2) * 8 + (i & 3) >= left) s[i] = 0.f;
    }
    acc.add(rd, KS0, s);
  };
  for (int t = 0; t < nk; t += 6) {
    tile(Stage<0>(), Stage<0>(), s0, s1, t);
    if (t + 1 < nk) tile(Stage<1>(), Stage<1>(), s1, s0, t + 1);
    if (t + 2 < nk) tile(Stage<2>(), Stage<0>(), s0, s1, t + 2);
    if (t + 3 < nk) tile(Stage<0>(), Stage<1>(), s1, s0, t + 3);
    if (t + 4 < nk) tile(Stage<1>(), Stage<0>(), s0, s1, t + 4);
    if (t + 5 < nk) tile(Stage<2>(), Stage<1>(), s1, s0, t + 5);
  }
  block_barrier();  // the output slots reuse the tile buffers
  acc.store(p.dqkv + static_cast<size_t>(first + q0) * ld + h * D, ld, 1.0f / sqrtf(static_cast<float>(D)), lane,
            (lds_char *)smem_raw + wid * 8192, len - q0);
}

// ------------------------------------------------------------------ backward: dK, dV
//
// Each wave owns 32 keys and keeps their K and V rows and both accumulators in
// registers.  Per tile of 32 queries: S = Q K^T and dP = dO V^T, P, dS, then
// dV^T += dO^T P and dK^T += Q^T dS, 32 products of 32x32x16 at D = 128 to 48
// full-rate vector instructions and 16 exponentials.  The accumulators of S and
// dP start from the dQ kernel's -lse sqrt(D) and -D_i, which lie in LDS in the
// order of the result's registers, so neither is subtracted afterwards.
//
// The three sets as for the forward: 897 us (1160 TFLOP/s), 128 (730), 293 (670;
// its longest workgroup takes 204 tiles in turn, four heads' 51, where all of them
// spread over the 512 that run at a time would be 106 each).  64 keys
// per wave, which would halve the LDS reads, leave one wave per SIMD and were
// slower; so was V in registers at D = 128 (spills).  Query tiles from the last
// down, which all of a sequence's workgroups would read together, gave nothing.

// LDS of one stage: the tiles of Q and dO, then -lse sqrt(D) and -D_i, for each of
// which a wave loads 64 values (a tile has 32).
constexpr int kDkvTiles = 2 * tile_bytes<32>(), kDkvStage = kDkvTiles + 2 * 64 * 4;

// Wide heads keep the V rows in LDS: K, V and the two accumulators would leave
// no registers to read operands ahead into.
constexpr bool dkdv_v_in_lds(int d) { return d > 80; }

template <int D, int WPE>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(WPE, WPE))) void
packed_bwd_dkdv_kernel(PackedAttnArgs p) {
  using H = Head<D>;
  constexpr int KT = 32, TB = tile_bytes<KT>(), TILES = kDkvTiles, STAGE = kDkvStage;  // Q, dO, vectors
  using Loads = PackedLoads<D, KT, 4>;
  constexpr bool VL = dkdv_v_in_lds(D);
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_char *)smem_raw));

  int item, kvh, first, len, row;
  packed_item(p.kv_heads, item, kvh);
  if (!load_item(p.plan, p.tokens, item, first, len, row)) return;
  // the list has a sequence's last rows first; with `causal` its first keys have
  // the most queries
  if (p.causal) row = max((len - 1) / kPackedRows * kPackedRows - row, 0);
  const int group = p.heads / p.kv_heads;
  const int A = p.heads * D, ld = A + 2 * p.kv_heads * D;
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int k0w = row + wid * 32;
  const bool active = k0w < len;  // wave-uniform
  const int key = k0w + (lane & 31);
  const bf16_t *seq = p.qkv + static_cast<size_t>(first) * ld;
  const bf16_t *dseq = p.dO + static_cast<size_t>(first) * A;

  // query tiles t0 .. nq - 1 of each of the group's heads in turn
  const int t0 = p.causal ? row / KT : 0, nq = (len + KT - 1) / KT;
  const int total = (nq - t0) * group;
  int ih = kvh * group, it = t0;  // head and tile issued next
  Loads lq, ld_o;
  lq.init(seq + static_cast<size_t>(t0) * KT * ld + ih * D, len - t0 * KT, ld, lds0, wid, lane, false);
  ld_o.init(dseq + static_cast<size_t>(t0) * KT * A + ih * D, len - t0 * KT, A, lds0 + TB, wid, lane, false);
  // wave 0 loads the tile's -lse sqrt(D), wave 1 its -D_i; past the sequence
  // they read as zero, as Q and dO do: P = 1 then meets zeros only
  const float *vecs = (wid == 0 ? p.nlse : p.ndvec) + first + t0 * KT;
  const uint32_t vec_lds = __builtin_amdgcn_readfirstlane(lds0 + TILES + (wid == 0 ? 0 : 256));
  const uint32_t vec_bytes = static_cast<uint32_t>(len - t0 * KT) * 4;
  u32x4_t rvec = make_rsrc(vecs + static_cast<size_t>(ih) * p.tokens, vec_bytes);
  uint32_t vec_off = 0;
  auto issue = [&](auto stage) {
    constexpr int ST = decltype(stage)::value * STAGE;
    lq.template issue<ST>();
    ld_o.template issue<ST>();
    if (wid < 2) issue_lds4<ST>(rvec, vec_lds, lane * 4, vec_off);
    vec_off += KT * 4;
    if (++it == nq) {
      it = t0, ++ih;
      lq.start(seq + static_cast<size_t>(t0) * KT * ld + ih * D, len - t0 * KT, ld);
      ld_o.start(dseq + static_cast<size_t>(t0) * KT * A + ih * D, len - t0 * KT, A);
      rvec = make_rsrc(vecs + static_cast<size_t>(ih) * p.tokens, vec_bytes);
      vec_off = 0;
    }
  };

  bf16x8_t kf[H::KS], vf[H::KS];
  const uint32_t vown = lds0 + 2 * STAGE + wid * (32 * D * 2) + lane * 16;  // this lane's V row, VL
  {
    const bf16_t *kp = seq + static_cast<size_t>(key) * ld + A + kvh * D;
    load_row_operand<D>(kf, kp, key < len, hf);
    load_row_operand<D>(vf, kp + p.kv_heads * D, key < len, hf);
    if constexpr (VL) {
#pragma unroll
      for (int kk = 0; kk < H::KS; ++kk)
        *reinterpret_cast<__attribute__((address_space(3))) bf16x8_t *>(vown + kk * 1024) = vf[kk];
    }
  }
  Result<D> dk, dv;
  dk.zero();
  dv.zero();
  const float c = kLog2e / sqrtf(static_cast<float>(D));
  PackedReads<D, true> rd;
  rd.init(lane, lds0);
  issue(Stage<0>());
  int ct = t0;  // the tile computed next
  auto tile = [&](auto stage, int n) {
    constexpr int ST = stage.value * STAGE;
    wait_vmcnt<0>();  // this wave's loads of tile n
    // every wave's loads of tile n have landed, and every wave is done with
    // tile n - 1, whose buffer is refilled next
    block_barrier();
    if (n + 1 < total) issue(Stage<1 - stage.value>());
    const int q0 = ct * KT;
    if (++ct == nq) ct = t0;
    // waves whose keys all lie past the sequence, or (causal) behind every
    // query of the tile, only load and synchronise
    if (!active || (p.causal && q0 + KT <= k0w)) return;
    rd.local();
    // register 4g + e is query 8g + 4 hf + e
    f32x16_t sl, dp;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4_t l4 = rd.vec(ST + TILES + g * 32), d4 = rd.vec(ST + TILES + 256 + g * 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) sl[4 * g + e] = l4[e], dp[4 * g + e] = d4[e];
    }
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk) sl = mfma32(rd.row(ST, 0, kk), kf[kk], sl);
#pragma unroll
    for (int kk = 0; kk < H::KS; ++kk)
      dp = mfma32(rd.row(ST + TB, 0, kk), VL ? rd.template at<bf16x8_t>(vown + kk * 1024) : vf[kk], dp);
#pragma unroll
    for (int i = 0; i < 16; ++i) sl[i] = exp2_hw(sl[i] * c);  // P
    if (p.causal && q0 < k0w + 31) {  // some query of the tile precedes some key of the wave
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (q0 + (i >> 2) * 8 + hf * 4 + (i & 3) < key) sl[i] = 0.f;
    }
    dv.add(rd, ST + TB, sl);
    dp *= sl;  // dS
    dk.add(rd, ST, dp);
  };
  for (int n = 0; n < total; n += 2) {
    tile(Stage<0>(), n);
    if (n + 1 < total) tile(Stage<1>(), n + 1);
  }
  block_barrier();  // the output slots reuse the tile buffers
  bf16_t *out = p.dqkv + static_cast<size_t>(first + k0w) * ld + A + kvh * D;
  lds_char *slot = (lds_char *)smem_raw + wid * 8192;
  dk.store(out, ld, 1.0f / sqrtf(static_cast<float>(D)), lane, slot, len - k0w);
  dv.store(out + p.kv_heads * D, ld, 1.0f, lane, slot, len - k0w);
}

// Waves per SIMD: as many as the registers of one allow.  LDS: the tiles' stages,
// which the waves' output slots of 8 KB reuse.
constexpr int kOutLds = 4 * 8192;

template <int D>
void launch_fwd_d(const PackedAttnArgs &a, hipStream_t s) {
  constexpr int lds = std::max(4 * tile_bytes<32>(), kOutLds), waves = D == 64 ? 4 : D == 80 ? 3 : 2;
  hipLaunchKernelGGL((packed_fwd_kernel<D, waves>), dim3(a.slots * a.heads), dim3(256), lds, s, a);
}

template <int D>
void launch_bwd_d(const PackedAttnArgs &a, hipStream_t s) {
  constexpr int dq_lds = std::max(5 * tile_bytes<32>(), kOutLds), dq_waves = D == 128 ? 2 : 3;
  constexpr int dkdv_lds = std::max(2 * kDkvStage + (dkdv_v_in_lds(D) ? 4 * 32 * D * 2 : 0), kOutLds);
  hipLaunchKernelGGL((packed_bwd_dq_kernel<D, dq_waves>), dim3(a.slots * a.heads), dim3(256), dq_lds, s, a);
  constexpr int dkdv_waves = D == 64 ? 3 : 2;
  hipLaunchKernelGGL((packed_bwd_dkdv_kernel<D, dkdv_waves>), dim3(a.slots * a.kv_heads), dim3(256), dkdv_lds, s, a);
}

PackedAttnArgs with_shared4(const PackedAttnArgs &args) {
  PackedAttnArgs a = args;
  a.shared4 = a.heads / a.kv_heads % 4 == 0;
  return a;
}

}  // namespace

bool launch_attn_packed_fwd(const PackedAttnArgs &args, hipStream_t s) {
  const PackedAttnArgs a = with_shared4(args);
  switch (a.d) {
    case 64: launch_fwd_d<64>(a, s); return true;
    case 80: launch_fwd_d<80>(a, s); return true;
    case 128: launch_fwd_d<128>(a, s); return true;
    default: return false;
  }
}

bool launch_attn_packed_bwd(const PackedAttnArgs &args, hipStream_t s) {
  const PackedAttnArgs a = with_shared4(args);
  switch (a.d) {
    case 64: launch_bwd_d<64>(a, s); return true;
    case 80: launch_bwd_d<80>(a, s); return true;
    case 128: launch_bwd_d<128>(a, s); return true;
    default: return false;
  }
}

}  // namespace optimus
