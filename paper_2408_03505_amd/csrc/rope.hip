// Rotary positions with up to three axes on the queries and keys of a packed
// qkv [M, (heads + 2 kv_heads) * D], columns [heads + 2 kv_heads][D].
//
// Pair i of every query and key vector is turned by pos[row, axis(i)] *
// inv_freq[i]; the backward turns it back (a rotation's transpose is its
// inverse), so one kernel serves both.  Pairs without an axis and the values are
// copied (the values not where the output is the input).
//
// Bound by memory: 4 bytes per element (read and written once) and one angle
// per row and pair, shared by all heads.  A workgroup takes one row: it
// computes the row's D / 2 angles into LDS once, while its first loads are
// under way, then streams the row in 16-byte chunks, a thread holding two
// chunks half a head apart (with "halves" pairs, the two members of eight
// pairs).  8192 rows of 144 heads of 128, 604 MB: 113 us, 5.3 TB/s, as fast as a
// large copy; 257 rows of 48 heads of 80: 3.2 us, a launch's own time.
#include "common.hpp"
#include "kernels.hpp"

namespace optimus {

namespace {

constexpr double kInvTwoPi = 0.15915494309189533577;

// cos and sin of pos * freq.  The product is formed in 64 bits and reduced to a
// fraction of a turn there: at position 10^6 a 32-bit angle would be off by up
// to 0.03 rad.  The fraction is then small enough for 32 bits (off by 2^-26
// turns at most).
__device__ __forceinline__ void angle_of(int pos, float freq, float &c, float &s) {
  double turns = static_cast<double>(pos) * static_cast<double>(freq) * kInvTwoPi;
  turns -= rint(turns);
  sincospif(2.0f * static_cast<float>(turns), &s, &c);
}

// (a, b) of one pair turned by the angle.
__device__ __forceinline__ void turn(float &a, float &b, float c, float s) {
  const float x = a * c - b * s;
  b = a * s + b * c;
  a = x;
}

template <int D, bool IL>
__global__ __launch_bounds__(256) void rope_kernel(int M, int qk_heads, int v_heads, int sec_t, int sec_th, int used,
                                                   const bf16_t *x, const int *__restrict__ pos,
                                                   const float *__restrict__ inv_freq, float sign, bf16_t *y) {
  constexpr int HALF = D / 2, CP = D / 16;  // pairs; chunk pairs per head
  __shared__ float cs[HALF], sn[HALF];
  const int tid = threadIdx.x;
  const int row = blockIdx.x;
  const size_t base = static_cast<size_t>(row) * (qk_heads + v_heads) * D;
  const int n = qk_heads * CP;
  // element offset of a chunk pair's first chunk
  auto at = [](int i) { return static_cast<size_t>(i / CP) * D + (i % CP) * 8; };
  u32x4_t lo{}, hi{};
  if (tid < n) {
    lo = ldg16(x + base + at(tid));
    hi = ldg16(x + base + at(tid) + HALF);
  }
  if (tid < used) {
    const int axis = tid < sec_t ? 0 : tid < sec_th ? 1 : 2;
    float c, s;
    angle_of(pos[static_cast<size_t>(row) * 3 + axis], inv_freq[tid], c, s);
    cs[tid] = c;
    sn[tid] = s * sign;
  }
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const u32x4_t a = lo, b = hi;
    if (i + 256 < n) {
      lo = ldg16(x + base + at(i + 256));
      hi = ldg16(x + base + at(i + 256) + HALF);
    }
    float p[8], q[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[2 * e] = lo_bf(a[e]), p[2 * e + 1] = hi_bf(a[e]);
      q[2 * e] = lo_bf(b[e]), q[2 * e + 1] = hi_bf(b[e]);
    }
    const int c8 = (i % CP) * 8;
    if constexpr (IL) {
      // pairs (2j, 2j + 1): four in each chunk
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = c8 / 2 + e;
        if (j < used) turn(p[2 * e], p[2 * e + 1], cs[j], sn[j]);
        if (j + HALF / 2 < used) turn(q[2 * e], q[2 * e + 1], cs[j + HALF / 2], sn[j + HALF / 2]);
      }
    } else {
      // pairs (j, j + D / 2): one member in each chunk
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c8 + e < used) turn(p[e], q[e], cs[c8 + e], sn[c8 + e]);
    }
    u32x4_t o0, o1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o0[e] = pack2(p[2 * e], p[2 * e + 1]);
      o1[e] = pack2(q[2 * e], q[2 * e + 1]);
    }
    stg16(y + base + at(i), o0);
    stg16(y + base + at(i) + HALF, o1);
  }
  if (x != y) {
    const size_t v0 = base + static_cast<size_t>(qk_heads) * D;
    for (int i = tid; i < v_heads * (D / 8); i += 256) stg16(y + v0 + i * 8, ldg16(x + v0 + i * 8));
  }
}

template <int D>
void rope_d(const RopeArgs &a, hipStream_t s) {
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(a.M), dim3(256), 0, s, a.M, a.heads + a.kv_heads, a.kv_heads, a.sec[0],
                       a.sec[0] + a.sec[1], a.sec[0] + a.sec[1] + a.sec[2], a.x, a.pos, a.inv_freq,
                       a.back ? -1.f : 1.f, a.y);
  };
  if (a.interleaved)
    go(rope_kernel<D, true>);
  else
    go(rope_kernel<D, false>);
}

}  // namespace

bool launch_rope(const RopeArgs &a, hipStream_t s) {
  switch (a.d) {
    case 64: rope_d<64>(a, s); return true;
    case 80: rope_d<80>(a, s); return true;
    case 128: rope_d<128>(a, s); return true;
    default: return false;
  }
}

}  // namespace optimus
