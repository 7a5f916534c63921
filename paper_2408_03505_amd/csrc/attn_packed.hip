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
//  - Every tile is loaded through a buffer resource of its own, which begins at
//    the tile's first row (64-bit, so a tensor may be as long as memory holds)
//    and ends with the sequence's last row: rows past it read as zero, and a
//    non-finite value behind a sequence never reaches it.  Lanes whose LDS
//    columns lie past the head's width ask for nothing.
//  - With `causal`, a query's keys end with itself: key tiles past a
//    workgroup's last query (query tiles before its first key, in dK/dV) are
//    skipped, and those on the diagonal are masked element by element.
//  - dK/dV runs over the queries of every head that shares the key head, in
//    head order, so the gradients of shared heads are summed in the
//    accumulators, with no atomics and always in the same order.
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
// the list holds; false past the list's end.
__device__ __forceinline__ bool load_item(const PackedPlan *plan, int slots, int tokens, int i, int &first, int &len,
                                          int &row) {
  if (i >= min(plan->count, slots)) return false;
  const PackedItem it = plan->item[i];
  first = __builtin_amdgcn_readfirstlane(min(max(it.first, 0), tokens));
  len = __builtin_amdgcn_readfirstlane(min(max(it.len, 0), tokens - first));
  row = __builtin_amdgcn_readfirstlane(max(it.row, 0));
  return row < len;
}

// Per-lane byte offsets of this wave's loads of a tile (rows ld elements
// apart); lanes past the head's width get one past every extent, which loads
// zero without touching memory.
template <int D, int KT, int NW, int N>
__device__ __forceinline__ void packed_voff(uint32_t (&v)[N], int wid, int lane, int ld, bool perm) {
  static_assert(N == TileLoads<KT, NW>::N, "one offset per load");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int o = (wid * N + i) * 1024 + lane * 16;
    const int pr = o >> 8, c = ((o & 255) >> 4) ^ tsw(pr);
    v[i] = c * 8 < D ? static_cast<uint32_t>(((perm ? perm23(pr) : pr) * ld + c * 8) * 2) : 0x80000000u;
  }
}

// Extent in bytes of `rows` rows from a head's first column, at most one tile.
template <int D, int KT>
__device__ __forceinline__ uint32_t tile_extent(int rows, int ld) {
  return static_cast<uint32_t>((min(rows, KT) - 1) * ld + D) * 2;
}

// Loads the tile at `src` (a head's first column in the tile's first row),
// `rows` rows of which are the sequence's.
template <int D, int KT, int NW, int N>
__device__ __forceinline__ void packed_issue(const bf16_t *src, int rows, int ld, uint32_t lds_tile,
                                             const uint32_t (&voff)[N], int wid) {
  const u32x4_t rsrc = make_rsrc(src, tile_extent<D, KT>(rows, ld));
#pragma unroll
  for (int i = 0; i < N; ++i)
    buffer_load_lds16(rsrc, __builtin_amdgcn_readfirstlane(lds_tile + (wid * N + i) * 1024), voff[i], 0);
}

// The two read patterns of a tile (TileReads) from whole LDS addresses, so that
// stage, tile, fragment and step all go in the reads' offset field, and reads
// of fp32 vectors in the order of a result's registers.  The tile swizzle is an
// XOR of the 16-byte chunk, so steps along the columns are an XOR of the first
// one's address: one vector instruction per read and two registers in all,
// where registers are what limits the kernel.
template <int D, bool PERM>
struct PackedReads {
  int row0, col0, vec0;
  __device__ __forceinline__ void init(int lane, uint32_t lds0) {
    row0 = lds0 + tile_off(lane & 31, lane >> 5);
    const int k = (PERM ? 4 : 8) * (lane >> 5) + ((lane & 15) >> 2);
    const int n = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    col0 = lds0 + tile_off(k, n >> 3) + (n & 7) * 2;
    vec0 = lds0 + (lane >> 5) * 16;
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
  // the second read: 8 rows further with PERM (tsw differs in one bit), else 4
  __device__ __forceinline__ bf16x8_t col(int base, int nf, int st) const {
    const int o = base + st * 16 * kDL * 2, c = col0 ^ (nf << 6);
    const int c1 = PERM ? (c ^ 32) + 8 * kDL * 2 : (c ^ 16) + 4 * kDL * 2;
    return lds_read_tr(reinterpret_cast<const lds_char *>(c + o), reinterpret_cast<const lds_char *>(c1 + o));
  }
  __device__ __forceinline__ f32x4_t vec(int base) const { return at<f32x4_t>(vec0 + base); }
};

// ------------------------------------------------------------------ forward

template <int D, int KT, int MINB>
__global__ __launch_bounds__(256, MINB) void packed_fwd_kernel(PackedAttnArgs p) {
  using H = Head<D>;
  constexpr int TB = tile_bytes<KT>(), NL = TileLoads<KT, 4>::N;
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];  // 2 x (K tile, V tile)
  const lds_char *smem = (const lds_char *)(smem_raw);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));

  int item, h, first, len, row;
  packed_item(p.heads, item, h);
  if (!load_item(p.plan, p.slots, p.tokens, item, first, len, row)) return;
  const int kvh = h / (p.heads / p.kv_heads);
  const int A = p.heads * D, ld = A + 2 * p.kv_heads * D;
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = row + wid * 32;  // the wave's first query
  const int q = q0 + (lane & 31);
  const bool active = q0 < len;  // wave-uniform
  const bf16_t *seq = p.qkv + static_cast<size_t>(first) * ld;
  const bf16_t *kp = seq + A + kvh * D, *vp = kp + p.kv_heads * D;

  uint32_t voff_k[NL], voff_v[NL];
  packed_voff<D, KT, 4>(voff_k, wid, lane, ld, false);
  packed_voff<D, KT, 4>(voff_v, wid, lane, ld, true);
  auto issue = [&](int t) {
    const uint32_t buf = lds0 + (t & 1) * 2 * TB;
    const size_t at = static_cast<size_t>(t) * KT * ld;
    packed_issue<D, KT, 4>(kp + at, len - t * KT, ld, buf, voff_k, wid);
    packed_issue<D, KT, 4>(vp + at, len - t * KT, ld, buf + TB, voff_v, wid);
  };

  bf16x8_t qf[H::KS];
  load_row_operand<D>(qf, seq + static_cast<size_t>(q) * ld + h * D, q < len, hf);

  f32x16_t acc[H::NF];
#pragma unroll
  for (int i = 0; i < H::NF; ++i) acc[i] = f32x16_t{};
  float m = -INFINITY, l = 0.f;
  const float c = kLog2e / sqrtf(static_cast<float>(D));

  TileReads<D, false> rd;
  rd.init(lane, 0, TB);
  // keys of the workgroup, of the wave, that all of the wave's queries see, and of this lane's query
  const int keys = p.causal ? min(len, row + kPackedRows) : len;
  const int wave_keys = !active ? 0 : p.causal ? min(len, q0 + 32) : len;
  const int all_see = p.causal ? q0 + 1 : len;
  const int lim = p.causal ? min(len, q + 1) : len;
  const int nk = (keys + KT - 1) / KT;
  issue(0);
  auto tile = [&](auto stage, int t) {
    wait_vmcnt<0>();  // this wave's loads of tile t have landed
    // every wave's loads of tile t have landed, and every wave is done with
    // tile t - 1, whose buffer the next issue refills
    block_barrier();
    if (t + 1 < nk) issue(t + 1);
    const lds_char *Ts = smem + stage.value * 2 * TB;
    const int k0 = t * KT;
    if (k0 < wave_keys) {  // waves that see none of the tile's keys only load and synchronise
      constexpr int NS = KT / 32;  // 32-key fragments per tile
      f32x16_t s[NS];
#pragma unroll
      for (int f = 0; f < NS; ++f) {
        s[f] = f32x16_t{};
#pragma unroll
        for (int kk = 0; kk < H::KS; ++kk) s[f] = mfma32(rd.row(Ts, f, kk), qf[kk], s[f]);
      }
      ColOperands<D, KT, (D <= kPrefetchMaxD), false> vop;  // V^T operands, read under the softmax
      vop.fetch(Ts, rd);
      if (k0 + KT > all_see) {
#pragma unroll
        for (int f = 0; f < NS; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k0 + f * 32 + (i >> 2) * 8 + hf * 4 + (i & 3) >= lim) s[f][i] = -INFINITY;
      }
      // Raw logits are scaled by c > 0, so the scaled maximum is c times the
      // raw one.  The reference maximum m of a query moves only when its
      // maximum exceeds m by more than kLazyRescale (log2 units): O = acc / l
      // and lse = m + log2 l hold for any m.  (Every query sees key 0, so m is
      // finite after the first tile.)
      float ms = -INFINITY;
#pragma unroll
      for (int f = 0; f < NS; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) ms = fmaxf(ms, s[f][i]);
      ms = fmaxf(ms, __shfl_xor(ms, 32, kWave));
      const float mt = ms * c;
      const bool grow = mt > m + kLazyRescale;
      if (__any(grow)) {
        const float mn = grow ? mt : m;
        const float alpha = exp2_hw(m - mn);  // 0 on the first tile (m = -inf), 1 where m stays
        m = mn;
        l *= alpha;
#pragma unroll
        for (int nf = 0; nf < H::NF; ++nf) acc[nf] *= alpha;
      }
      float ls = 0.f;
#pragma unroll
      for (int f = 0; f < NS; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float pv = exp2_hw(__builtin_fmaf(s[f][i], c, -m));
          s[f][i] = pv;
          ls += pv;
        }
      l += ls;
#pragma unroll
      for (int st = 0; st < KT / 16; ++st) {
        const bf16x8_t pb = pack8(s[st >> 1], st & 1);
#pragma unroll
        for (int nf = 0; nf < H::NF; ++nf) acc[nf] = mfma32(vop.get(Ts, rd, nf, st), pb, acc[nf]);
      }
    }
  };
  for (int t = 0; t < nk; t += 2) {
    tile(Stage<0>(), t);
    if (t + 1 < nk) tile(Stage<1>(), t + 1);
  }
  block_barrier();  // every wave is done with the tile buffers, which the output slots reuse

  const float lt = l + __shfl_xor(l, 32, kWave);
  if (q < len && hf == 0) p.lse[static_cast<size_t>(h) * p.tokens + first + q] = (m + log2f(lt)) / kLog2e;
  store_dmajor_lds<D>(p.o + static_cast<size_t>(first + q0) * A + h * D, A, acc, 1.0f / lt, lane,
                      const_cast<lds_char *>(smem) + wid * 8192, len - q0);
}

// ------------------------------------------------------------------ backward: dQ and D

template <int D, int NW, int KT, int MINB>
__global__ __launch_bounds__(NW * 64, MINB) void packed_bwd_dq_kernel(PackedAttnArgs p) {
  using H = Head<D>;
  static_assert(32 * NW == kPackedRows, "one item per workgroup");
  constexpr int TB = tile_bytes<KT>(), NL = TileLoads<KT, NW>::N, STAGE = 2 * TB;  // K, V
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const lds_char *smem = (const lds_char *)(smem_raw);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));

  int item, h, first, len, row;
  packed_item(p.heads, item, h);
  if (!load_item(p.plan, p.slots, p.tokens, item, first, len, row)) return;
  const int kvh = h / (p.heads / p.kv_heads);
  const int A = p.heads * D, ld = A + 2 * p.kv_heads * D;
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = row + wid * 32, q = q0 + (lane & 31);
  const bool qvalid = q < len, active = q0 < len;
  const bf16_t *seq = p.qkv + static_cast<size_t>(first) * ld;
  const bf16_t *kp = seq + A + kvh * D, *vp = kp + p.kv_heads * D;
  const size_t orow = static_cast<size_t>(first + q) * A + h * D;
  const size_t vec = static_cast<size_t>(h) * p.tokens + first + q;

  uint32_t voff[NL];
  packed_voff<D, KT, NW>(voff, wid, lane, ld, false);
  auto issue = [&](int t) {
    const uint32_t buf = lds0 + (t & 1) * STAGE;
    const size_t at = static_cast<size_t>(t) * KT * ld;
    packed_issue<D, KT, NW>(kp + at, len - t * KT, ld, buf, voff, wid);
    packed_issue<D, KT, NW>(vp + at, len - t * KT, ld, buf + TB, voff, wid);
  };

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

  f32x16_t acc[H::NF];
#pragma unroll
  for (int i = 0; i < H::NF; ++i) acc[i] = f32x16_t{};
  constexpr int NS = KT / 32;  // 32-key fragments per tile
  const int keys = p.causal ? min(len, row + kPackedRows) : len;
  const int wave_keys = !active ? 0 : p.causal ? min(len, q0 + 32) : len;
  const int all_see = p.causal ? q0 + 1 : len;
  const int lim = p.causal ? min(len, q + 1) : len;
  const int nk = (keys + KT - 1) / KT;
  // K: row reads for S^T and the permuted column reads; V (TB further): row reads
  TileReads<D, true> rd;
  rd.init(lane, 0, 0);
  issue(0);
  auto tile = [&](auto stage, int t) {
    wait_vmcnt<0>();  // this wave's loads of tile t
    block_barrier();  // everyone's loads of tile t landed; tile t - 1's buffer is free
    if (t + 1 < nk) issue(t + 1);
    const lds_char *Ks = smem + stage.value * STAGE, *Vs = Ks + TB;
    const int k0 = t * KT;
    if (k0 < wave_keys) {  // waves that see none of the tile's keys only load and synchronise
      f32x16_t sv[NS], dp[NS];
#pragma unroll
      for (int f = 0; f < NS; ++f) {
        sv[f] = f32x16_t{};
        dp[f] = f32x16_t{};
#pragma unroll
        for (int kk = 0; kk < H::KS; ++kk) {
          sv[f] = mfma32(rd.row(Ks, f, kk), qf[kk], sv[f]);
          dp[f] = mfma32(rd.row(Vs, f, kk), df[kk], dp[f]);
        }
      }
#pragma unroll
      for (int f = 0; f < NS; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sv[f][i] = exp2_hw(__builtin_fmaf(sv[f][i], c, -lse2)) * (dp[f][i] - dd);  // dS^T
      if (k0 + KT > all_see) {
        // register i of fragment f is key k0 + f*32 + 8(i/4) + 4 hf + i%4
#pragma unroll
        for (int f = 0; f < NS; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k0 + f * 32 + (i >> 2) * 8 + hf * 4 + (i & 3) >= lim) sv[f][i] = 0.f;
      }
#pragma unroll
      for (int st = 0; st < KT / 16; ++st) {
        const bf16x8_t sb = pack8(sv[st >> 1], st & 1);
#pragma unroll
        for (int nf = 0; nf < H::NF; ++nf) acc[nf] = mfma32(rd.col(Ks, nf, st), sb, acc[nf]);
      }
    }
  };
  for (int t = 0; t < nk; t += 2) {
    tile(Stage<0>(), t);
    if (t + 1 < nk) tile(Stage<1>(), t + 1);
  }
  block_barrier();  // the output slots reuse the tile buffers
  store_dmajor_lds<D>(p.dqkv + static_cast<size_t>(first + q0) * ld + h * D, ld, acc,
                      1.0f / sqrtf(static_cast<float>(D)), lane, const_cast<lds_char *>(smem) + wid * 8192, len - q0);
}

// ------------------------------------------------------------------ backward: dK, dV
//
// Each wave owns 32 keys and keeps their K and V rows and both accumulators in
// registers.  Per tile of 32 queries: S = Q K^T and dP = dO V^T, P, dS, then
// dV^T += dO^T P and dK^T += Q^T dS, 32 products of 32x32x16 at D = 128 to 48
// full-rate vector instructions and 16 exponentials.  The accumulators of S and
// dP start from the dQ kernel's -lse sqrt(D) and -D_i, which lie in LDS in the
// order of the result's registers, so neither is subtracted afterwards.

// LDS of one stage: the Q and dO tiles, then -lse sqrt(D) and -D_i of up to 64 queries.
template <int KT>
constexpr int packed_dkdv_stage() {
  return 2 * tile_bytes<KT>() + 2 * 64 * 4;
}

// Wide heads keep the V rows in LDS: K, V and the two accumulators would leave
// no registers to read operands ahead into.
constexpr bool dkdv_v_in_lds(int d) { return d > 80; }

template <int D, int NW, int KT, int MINB>
__global__ __launch_bounds__(NW * 64, MINB) void packed_bwd_dkdv_kernel(PackedAttnArgs p) {
  using H = Head<D>;
  static_assert(32 * NW == kPackedRows, "one item per workgroup");
  constexpr int TB = tile_bytes<KT>(), NL = TileLoads<KT, NW>::N, TILES = 2 * TB;  // Q, dO
  constexpr int STAGE = packed_dkdv_stage<KT>(), NS = KT / 32;
  constexpr bool VL = dkdv_v_in_lds(D);
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const lds_char *smem = (const lds_char *)(smem_raw);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));

  int item, kvh, first, len, row;
  packed_item(p.kv_heads, item, kvh);
  if (!load_item(p.plan, p.slots, p.tokens, item, first, len, row)) return;
  const int group = p.heads / p.kv_heads;
  const int A = p.heads * D, ld = A + 2 * p.kv_heads * D;
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int k0w = row + wid * 32;
  const bool active = k0w < len;  // wave-uniform
  const int key = k0w + (lane & 31);
  const bf16_t *seq = p.qkv + static_cast<size_t>(first) * ld;
  const bf16_t *dseq = p.dO + static_cast<size_t>(first) * A;

  // Two loads per tile and wave, the second four rows further, where the swizzle
  // swaps neighbouring chunks: its offset is made from the first one's when it
  // is needed (rows are multiples of 32 bytes).
  static_assert(NL == 2, "two loads per tile and wave");
  uint32_t v0[NL];
  packed_voff<D, KT, NW>(v0, wid, lane, ld, false);
  const uint32_t vq = v0[0];
  packed_voff<D, KT, NW>(v0, wid, lane, A, false);
  const uint32_t vd = v0[0];
  auto load2 = [&](const bf16_t *src, int rows, int rld, uint32_t lds_tile, uint32_t v) {
    const uint32_t both[2] = {v, (v ^ 16) + static_cast<uint32_t>(8 * rld)};
    packed_issue<D, KT, NW>(src, rows, rld, lds_tile, both, wid);
  };
  // query tiles t0 .. nq - 1 of each of the group's heads in turn
  const int t0 = p.causal ? row / KT : 0, nq = (len + KT - 1) / KT;
  const int total = (nq - t0) * group;
  int ih = kvh * group, it = t0;  // head and tile issued next
  auto issue = [&](int n) {
    const uint32_t buf = lds0 + (n & 1) * STAGE;
    const int rem = len - it * KT;
    load2(seq + static_cast<size_t>(it) * KT * ld + ih * D, rem, ld, buf, vq);
    load2(dseq + static_cast<size_t>(it) * KT * A + ih * D, rem, A, buf + TB, vd);
    // the tile's vectors; past the sequence they read as zero, as Q and dO do:
    // P = 1 then meets zeros only
    const size_t vec = static_cast<size_t>(ih) * p.tokens + first + it * KT;
    const uint32_t ext = static_cast<uint32_t>(min(rem, KT)) * 4;
    if (wid == 0)
      buffer_load_lds4(make_rsrc(p.nlse + vec, ext), __builtin_amdgcn_readfirstlane(buf + TILES), lane * 4, 0);
    if (wid == 1)
      buffer_load_lds4(make_rsrc(p.ndvec + vec, ext), __builtin_amdgcn_readfirstlane(buf + TILES + 64 * 4), lane * 4,
                       0);
    if (++it == nq) it = t0, ++ih;
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
  f32x16_t dk[H::NF], dv[H::NF];
#pragma unroll
  for (int i = 0; i < H::NF; ++i) dk[i] = f32x16_t{}, dv[i] = f32x16_t{};
  const float c = kLog2e / sqrtf(static_cast<float>(D));
  PackedReads<D, true> rd;
  rd.init(lane, lds0);
  issue(0);
  int ct = t0;  // the tile computed next
  auto tile = [&](auto stage, int n) {
    constexpr int ST = stage.value * STAGE;
    wait_vmcnt<0>();  // this wave's loads of tile n
    // every wave's loads of tile n have landed, and every wave is done with
    // tile n - 1, whose buffer is refilled next
    block_barrier();
    if (n + 1 < total) issue(n + 1);
    const int q0 = ct * KT;
    if (++ct == nq) ct = t0;
    // waves whose keys all lie past the sequence, or (causal) behind every
    // query of the tile, only load and synchronise
    if (!active || (p.causal && q0 + KT <= k0w)) return;
    rd.local();
    // register 4g+e of fragment f is query f*32 + 8g + 4hf + e
    f32x16_t s[NS], dp[NS];
#pragma unroll
    for (int f = 0; f < NS; ++f) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t l4 = rd.vec(ST + TILES + f * 128 + g * 32), d4 = rd.vec(ST + TILES + 256 + f * 128 + g * 32);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[f][4 * g + e] = l4[e], dp[f][4 * g + e] = d4[e];
      }
#pragma unroll
      for (int kk = 0; kk < H::KS; ++kk) s[f] = mfma32(rd.row(ST, f, kk), kf[kk], s[f]);
#pragma unroll
      for (int kk = 0; kk < H::KS; ++kk)
        dp[f] = mfma32(rd.row(ST + TB, f, kk), VL ? rd.template at<bf16x8_t>(vown + kk * 1024) : vf[kk], dp[f]);
    }
#pragma unroll
    for (int f = 0; f < NS; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[f][i] = exp2_hw(s[f][i] * c);  // P
    if (p.causal && q0 < k0w + 31) {  // some query of the tile precedes some key of the wave
#pragma unroll
      for (int f = 0; f < NS; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (q0 + f * 32 + (i >> 2) * 8 + hf * 4 + (i & 3) < key) s[f][i] = 0.f;
    }
#pragma unroll
    for (int st = 0; st < KT / 16; ++st) {
      const bf16x8_t pb = pack8(s[st >> 1], st & 1);
#pragma unroll
      for (int nf = 0; nf < H::NF; ++nf) dv[nf] = mfma32(rd.col(ST + TB, nf, st), pb, dv[nf]);
    }
#pragma unroll
    for (int f = 0; f < NS; ++f) dp[f] *= s[f];  // dS
#pragma unroll
    for (int st = 0; st < KT / 16; ++st) {
      const bf16x8_t sb = pack8(dp[st >> 1], st & 1);
#pragma unroll
      for (int nf = 0; nf < H::NF; ++nf) dk[nf] = mfma32(rd.col(ST, nf, st), sb, dk[nf]);
    }
  };
  for (int n = 0; n < total; n += 2) {
    tile(Stage<0>(), n);
    if (n + 1 < total) tile(Stage<1>(), n + 1);
  }
  block_barrier();  // the output slots reuse the tile buffers
  bf16_t *out = p.dqkv + static_cast<size_t>(first + k0w) * ld + A + kvh * D;
  lds_char *slot = const_cast<lds_char *>(smem) + wid * 8192;
  store_dmajor_lds<D>(out, ld, dk, 1.0f / sqrtf(static_cast<float>(D)), lane, slot, len - k0w);
  store_dmajor_lds<D>(out + p.kv_heads * D, ld, dv, 1.0f, lane, slot, len - k0w);
}

// Launch shapes: 4 waves of 32 queries (forward, dQ) or keys (dK/dV); KT is the
// token tile streamed through LDS, MINB the workgroups each CU must hold at once.
constexpr int kFwdKT = 32, kFwdMinBlocks = 3, kFwdSmallGrid = 256;
constexpr int kDqWaves = 4, kDqKT = 32, kDqMinBlocks = 2;
constexpr int kDkvWaves = 4, kDkvKT = 32, kDkvMinBlocks = 2;

template <int D, int KT, int MINB>
void launch_fwd_cfg(const PackedAttnArgs &a, hipStream_t s) {
  // two stages of (K, V) tiles; the per-wave 8 KB output slots reuse them
  constexpr int lds = std::max(4 * tile_bytes<KT>(), 4 * 8192);
  hipLaunchKernelGGL((packed_fwd_kernel<D, KT, MINB>), dim3(a.slots * a.heads), dim3(256), lds, s, a);
}

// A grid that leaves CUs idle runs each workgroup's tiles back to back with
// nothing else on the CU to hide their latency: there fewer, longer tiles win.
template <int D>
void launch_fwd_d(const PackedAttnArgs &a, hipStream_t s) {
  if (static_cast<long>(a.slots) * a.heads <= kFwdSmallGrid)
    launch_fwd_cfg<D, 64, 2>(a, s);
  else
    launch_fwd_cfg<D, kFwdKT, kFwdMinBlocks>(a, s);
}

template <int D>
void launch_bwd_d(const PackedAttnArgs &a, hipStream_t s) {
  constexpr int kDqLds = std::max(4 * tile_bytes<kDqKT>(), kDqWaves * 8192);
  constexpr int kDkvLds =
      std::max(2 * packed_dkdv_stage<kDkvKT>() + (dkdv_v_in_lds(D) ? kDkvWaves * 32 * D * 2 : 0), kDkvWaves * 8192);
  hipLaunchKernelGGL((packed_bwd_dq_kernel<D, kDqWaves, kDqKT, kDqMinBlocks>), dim3(a.slots * a.heads),
                     dim3(kDqWaves * 64), kDqLds, s, a);
  hipLaunchKernelGGL((packed_bwd_dkdv_kernel<D, kDkvWaves, kDkvKT, kDkvMinBlocks>), dim3(a.slots * a.kv_heads),
                     dim3(kDkvWaves * 64), kDkvLds, s, a);
}

}  // namespace

bool launch_attn_packed_fwd(const PackedAttnArgs &a, hipStream_t s) {
  switch (a.d) {
    case 64: launch_fwd_d<64>(a, s); return true;
    case 80: launch_fwd_d<80>(a, s); return true;
    case 128: launch_fwd_d<128>(a, s); return true;
    default: return false;
  }
}

bool launch_attn_packed_bwd(const PackedAttnArgs &a, hipStream_t s) {
  switch (a.d) {
    case 64: launch_bwd_d<64>(a, s); return true;
    case 80: launch_bwd_d<80>(a, s); return true;
    case 128: launch_bwd_d<128>(a, s); return true;
    default: return false;
  }
}

}  // namespace optimus
