// RMSNorm with the residual's addition and per-token quantisation of its output.
//
//   h = store(x + residual)          (x itself without a residual; store rounds to the element type)
//   r = fl32(1 / sqrt(mean(h^2) + eps))   mean and root in float64
//   y = fl32(fl32(h r) gain)
//   s = fl32(fl32(clip max|y|) / (2^(k-1) - 1)),  code = clamp(rint(fl32(y / s))),  value = store(fl32(code s))
//
// One pass over the data: a row stays in registers between the sum of squares and the codes.  What bounds it is HBM
// (7 bytes an entry with a bf16 residual and codes); a row of up to 1024 entries belongs to one warp or a part of
// it (no block barrier), a wider one to a block of up to 1024 threads that hold 16 or 32 entries each.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace kt {

// The serving kernels may be placed while the kernel before them in the stream still runs (a programmatic launch): their
// first act is to wait until all that came before is complete and visible.  A launch's own latency is hidden that way.
__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// An ordinary load: unlike __ldg, whose memory the compiler may take for constant, it stays behind that wait.
template <typename T>
__device__ __forceinline__ T plain_load(const T* p) { return *p; }

struct NormParams {
  const void* x;
  const void* res;     // null: no residual
  void* sum;           // null: x + residual is not stored
  const float* gain;   // null: unit gain
  int8_t* codes;       // null: no codes
  float* scales;       // null only when bits == 0
  void* values;        // null: no values
  long long ldx, ldr, lds, ldv;
  int rows, d;
  int bits;            // 0: values are y itself
  int values_f32;
  int ahead;           // groups may begin in front of the row (not VEC)
  float clip, den;
  double eps;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
  v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(p + 4), make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                            pack_bf16(v[6], v[7])));
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
// fl32(1 / sqrt(a)), 0 for 0: the float32 estimate (2 ulp) refined by two Newton steps in float64 (error
// below 2^-40), for a tenth of the float64 division and root.  Outside float32's comfortable range the plain form.
__device__ __forceinline__ float inv_sqrt_rn(double a) {
  if (a > 1e-30 && a < 1e30) {
    double r = static_cast<double>(rsqrtf(static_cast<float>(a)));
    r = r * (1.5 - 0.5 * a * r * r);
    r = r * (1.5 - 0.5 * a * r * r);
    return static_cast<float>(r);
  }
  return a == 0.0 ? 0.f : static_cast<float>(1.0 / sqrt(a));  // (a row of zeros without eps: factor 0)
}

// off + rint(fl32(t / s)) of eight entries, clamped to [lo, hi] + off, for s > 0 and without a division for nearly every
// entry.  off is 0 or a power of two (where code zero is held).  t fl32(1/s) + off is within 1e-4 of the quotient plus
// off while that is below 256, so only a quotient nearer than that to a border between two codes needs the division
// itself (one in 5000; the eight are then all divided).  Adding 1.5 2^23 rounds to an integer (ties to even, and off is
// even) and leaves the result in the low bits of the sum: bits[e] mod 2^22, two's complement.  `divide`: 1/s is out of
// range, always divide.  clamp == false: the quotients are known to round into [lo, hi] (a range that was not clipped).
constexpr float kRoundMagic = 12582912.f;
__device__ __forceinline__ bool quant_needs_division(float s) { return !(s > 1e-30f && s < 1e30f); }
__device__ __forceinline__ void quant8(const float (&t)[8], float s, float inv, bool divide, bool clamp, float lo,
                                       float hi, float off, float (&r)[8], uint32_t (&bits)[8]) {
  float far = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float q = __fmaf_rn(t[e], inv, off);
    if (clamp) q = fminf(fmaxf(q, lo + off), hi + off);
    const float m = __fadd_rn(q, kRoundMagic);
    bits[e] = __float_as_uint(m);
    r[e] = __fsub_rn(m, kRoundMagic);
    far = fmaxf(far, fabsf(__fsub_rn(q, r[e])));
  }
  if (divide || far > 0.4999f) {
#pragma unroll 1
    for (int e0 = 0; e0 < 2; ++e0) {
#pragma unroll
      for (int e1 = 0; e1 < 4; ++e1) {
        const float x = e0 ? t[4 + e1] : t[e1];
        const float v = fminf(fmaxf(rintf(__fdiv_rn(x, s)), lo), hi) + off;
        const uint32_t w = __float_as_uint(__fadd_rn(v, kRoundMagic));
        if (e0) r[4 + e1] = v, bits[4 + e1] = w;
        else r[e1] = v, bits[e1] = w;
      }
    }
  }
}
// the low bytes of four words
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// two entries as the element type holds them
__device__ __forceinline__ void stored2(float& a, float& b, const float*) {}
__device__ __forceinline__ void stored2(float& a, float& b, const __nv_bfloat16*) {
  const uint32_t w = pack_bf16(a, b);
  a = bf16_lo(w);
  b = bf16_hi(w);
}

// Eight entries of a row from j0 on, whatever their alignment, entries outside 0 .. d - 1 as zeros: the aligned 16-byte
// pieces that hold them (a piece that holds none of the row is not read), shifted into place.  The shift is the same for
// all groups of a row.  (A row's first and last piece may hold up to 14 bytes of what lies beside it: read, never used.)
template <typename T>
__device__ __forceinline__ void load8_any(const T* row, int j0, int d, float (&v)[8]) {
  constexpr int N = sizeof(T) / 2 + 1;  // pieces
  const uintptr_t first = reinterpret_cast<uintptr_t>(row), last = reinterpret_cast<uintptr_t>(row + d);
  const uintptr_t from = reinterpret_cast<uintptr_t>(row + j0), base = from & ~static_cast<uintptr_t>(15);
  uint32_t w[4 * N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint4 q = make_uint4(0u, 0u, 0u, 0u);
    const uintptr_t at = base + 16 * i;
    if (at + 16 > first && at < last) q = *reinterpret_cast<const uint4*>(at);
    w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
  }
  const uint32_t by = static_cast<uint32_t>(from) & 15u;
  if (by & 8u) {
#pragma unroll
    for (int i = 0; i + 2 < 4 * N; ++i) w[i] = w[i + 2];
  }
  if (by & 4u) {
#pragma unroll
    for (int i = 0; i + 3 < 4 * N; ++i) w[i] = w[i + 1];
  }
  if constexpr (sizeof(T) == 2) {
    if (by & 2u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  }
  if (j0 < 0 || j0 + 8 > d) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j0 + e < 0 || j0 + e >= d) v[e] = 0.f;
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void load_group(const T* row, int j0, int d, float (&v)[8]) {
  if constexpr (VEC) load8(row + j0, v);
  else load8_any(row, j0, d, v);
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_group(T* row, int j0, int d, const float (&v)[8]) {
  if (VEC || (j0 >= 0 && j0 + 8 <= d && (reinterpret_cast<uintptr_t>(row + j0) & 15u) == 0)) {
    store8(row + j0, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j0 + e >= 0 && j0 + e < d) store1(row + j0 + e, v[e]);
  }
}
template <bool VEC>
__device__ __forceinline__ void put_values(const NormParams& p, long long row, int j0, const float (&q)[8]) {
  if (p.values_f32) store_group<VEC>(static_cast<float*>(p.values) + row * p.ldv, j0, p.d, q);
  else store_group<VEC>(static_cast<__nv_bfloat16*>(p.values) + row * p.ldv, j0, p.d, q);
}

// T: element type.  V: groups of eight entries a thread holds.  VEC: rows are 16-byte aligned and d is a multiple of
// 8; else a row's groups begin `ahead` entries before it, so that (nearly all of) the first output's are aligned: loads of
// any alignment are two or three aligned ones and a shift, stores of another alignment than that output's go entry by
// entry (8000 rows of 4097 with residual and codes 96 us; all of it entry by entry 166 us).  LANES: lanes that share a row,
// 0 for a row per block.
template <typename T, int V, bool VEC, int LANES>
__global__ void __launch_bounds__(LANES > 0 ? 128 : 1024) k_rmsnorm_quant(const NormParams p) {
  __shared__ double sh_sum[32];
  __shared__ unsigned int sh_max[32];
  wait_for_earlier_kernels();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr bool kShared = LANES > 0;
  const int nthr = kShared ? LANES : blockDim.x;
  const int tid = kShared ? threadIdx.x % nthr : threadIdx.x;
  long long row = kShared ? static_cast<long long>(blockIdx.x) * (blockDim.x / nthr) + threadIdx.x / nthr : blockIdx.x;
  const bool mine = !kShared || row < p.rows;
  if (!mine) row = p.rows - 1;  // (lanes without a row take the last one's, and store nothing)
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  const T* res = p.res ? static_cast<const T*>(p.res) + row * p.ldr : nullptr;
  T* sum = p.sum && mine ? static_cast<T*>(p.sum) + row * p.lds : nullptr;
  const int d = p.d;

  int ahead = 0;
  if (!VEC && p.ahead) {
    if (p.codes != nullptr) ahead = static_cast<int>(reinterpret_cast<uintptr_t>(p.codes + row * d) & 7u);
    else if (p.values_f32) ahead = static_cast<int>(reinterpret_cast<uintptr_t>(static_cast<float*>(p.values) + row * p.ldv) / 4 & 7u);
    else ahead = static_cast<int>(reinterpret_cast<uintptr_t>(static_cast<__nv_bfloat16*>(p.values) + row * p.ldv) / 2 & 7u);
  }
  const int groups = VEC ? d >> 3 : (d + ahead + 7) >> 3;

  float h[V][8];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int v = tid + k * nthr;
    if (v < groups) {
      load_group<VEC>(x, 8 * v - ahead, d, h[k]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) h[k][e] = 0.f;
    }
  }
  if (res != nullptr) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int v = tid + k * nthr;
      if (v < groups) {
        float r[8];
        load_group<VEC>(res, 8 * v - ahead, d, r);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          h[k][e] = __fadd_rn(h[k][e], r[e]);
          h[k][e + 1] = __fadd_rn(h[k][e + 1], r[e + 1]);
          stored2(h[k][e], h[k][e + 1], x);
        }
        if (sum != nullptr) store_group<VEC>(sum, 8 * v - ahead, d, h[k]);
      }
    }
  }

  // the mean square in float64: the factor r is then the same float32 whatever the order of the sum
  double ss = 0.0;
#pragma unroll
  for (int k = 0; k < V; ++k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double a = static_cast<double>(h[k][e]);
      ss = fma(a, a, ss);
    }
  }
#pragma unroll
  for (int o = kShared ? LANES / 2 : 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if constexpr (!kShared) {
    if (lane == 0) sh_sum[warp] = ss;
    __syncthreads();
    ss = 0.0;
    for (int w = 0; w < (nthr >> 5); ++w) ss += sh_sum[w];
  }
  const float r = inv_sqrt_rn(ss / d + p.eps);

  // max|y|.  A NaN or an infinity of h shows in the mean square, an overflow of y in the maximum; a gain that is no
  // number is looked for.
  float top = 0.f;
  bool odd = !(ss < __longlong_as_double(0x7ff0000000000000ll));
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float g[8];
    if (p.gain != nullptr) {
      const int v = tid + k * nthr;
      if (v >= groups) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = 0.f;
      } else if (VEC && (reinterpret_cast<uintptr_t>(p.gain) & 15u) == 0) {
        load8(p.gain + 8 * v, g);
      } else {
        load8_any(p.gain, 8 * v - ahead, d, g);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y = __fmul_rn(h[k][e], r);
      if (p.gain != nullptr) {
        y = __fmul_rn(y, g[e]);
        odd |= !(fabsf(g[e]) < __uint_as_float(0x7f800000u));
      }
      h[k][e] = y;
      top = fmaxf(top, fabsf(y));
    }
  }
  if (p.bits == 0) {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (mine && tid + k * nthr < groups) put_values<VEC>(p, row, 8 * (tid + k * nthr) - ahead, h[k]);
    return;
  }
  // (the maximum of magnitudes is that of their bit patterns)
  unsigned int topb = odd ? 0x7f800000u : __float_as_uint(top);
  if constexpr (kShared && LANES < 32) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) topb = max(topb, __shfl_xor_sync(0xffffffffu, topb, o));
  } else {
    topb = __reduce_max_sync(0xffffffffu, topb);
  }
  if constexpr (!kShared) {
    if (lane == 0) sh_max[warp] = topb;
    __syncthreads();
    topb = 0u;
    for (int w = 0; w < (nthr >> 5); ++w) topb = max(topb, sh_max[w]);
  }
  const bool bad = topb >= 0x7f800000u;  // a row with an infinity or a NaN: scale and values NaN, codes 0
  const float s = bad ? __uint_as_float(0x7fc00000u) : __fdiv_rn(__fmul_rn(p.clip, __uint_as_float(topb)), p.den);
  if (!mine) return;
  if (tid == 0) p.scales[row] = s;
  const bool divide = quant_needs_division(s), clamp = p.clip != 1.f;
  const float inv = divide ? 0.f : __frcp_rn(s);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float q[8];
    uint32_t w[8];
    if (s > 0.f) {
      quant8(h[k], s, inv, divide, clamp, -p.den, p.den, 0.f, q, w);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = 0.f, w[e] = 0u;
    }
    const int v = tid + k * nthr, j0 = 8 * v - ahead;
    if (v >= groups) continue;
    if (p.codes != nullptr) {
      int8_t* c = p.codes + row * d + j0;
      if (VEC || (j0 >= 0 && j0 + 8 <= d && (reinterpret_cast<uintptr_t>(c) & 7u) == 0)) {
        *reinterpret_cast<uint2*>(c) =
            make_uint2(pack_bytes(w[0], w[1], w[2], w[3]), pack_bytes(w[4], w[5], w[6], w[7]));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (j0 + e >= 0 && j0 + e < d) c[e] = static_cast<int8_t>(w[e] & 0xffu);
      }
    }
    if (p.values != nullptr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = __fmul_rn(q[e], s);
      put_values<VEC>(p, row, j0, q);
    }
  }
}

}  // namespace kt
