// The paged, quantised KV cache: its layout, and the append that fills it.
//
// codes  [pages][heads][page_size][head_dim * bits / 8] uint8   4-bit codes: entry 2i in the low half of byte i
// steps  [pages][heads][page_size][2] float32                   (scale, shift) of a token's head
// A held entry stands for fl32(fl32(scale u) + shift), u its code from zero upwards; the symmetric quantizer's code c is
// held as u = c + 2^(k-1) with shift = -2^(k-1) scale, so readers need not know which quantizer wrote the cache.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "serve_norm.cuh"

namespace kt {

struct CacheView {
  uint8_t *k_codes, *v_codes;
  float2 *k_steps, *v_steps;
  int pages, heads, page_shift;  // page_size = 1 << page_shift
};

struct BatchView {
  const int *row_starts, *lengths, *page_table;
  int n_seqs, table_ld, max_rows, max_length;
};

struct AppendParams {
  CacheView c;
  BatchView b;
  const void *q, *k, *v;  // q null: keys and values only
  long long ldq, ldk, ldv;
  __nv_bfloat16 *q_out, *k_values, *v_values;  // values null: not wanted
  long long ldqo, ldkv, ldvv;
  const float* rope;  // [rope_rows][head_dim / 2][2] cosine, sine; null: no rotary positions
  int rope_rows;
  int rows, q_heads;
  int tokens;  // rows a block appends
  int hadamard, asym;
  float clip, den;  // den: 2^k - 1 or 2^(k-1) - 1
  float had_scale;  // fl32(1 / sqrt(head_dim))
  unsigned int* err;
};

constexpr unsigned int kCacheErrBatch = 1;  // row_starts, lengths or positions out of their bounds
constexpr unsigned int kCacheErrPage = 2;   // a page id out of range

// The sequence s with row_starts[s] = begin <= row < end = row_starts[s + 1], found by the whole warp in steps of 32; -1 if
// there is none (rows in front of the first sequence or behind the last, or starts that do not ascend).
__device__ __forceinline__ int find_sequence(const int* row_starts, int n_seqs, int row, int* begin, int* end) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_seqs;  // the candidates are lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + 31) >> 5;
    const int i = lo + (lane + 1) * step;  // first candidate of the next part
    const bool below = (lane + 1) * step < n && plain_load(row_starts + i) <= row;
    const int part = __popc(__ballot_sync(0xffffffffu, below));
    lo += part * step;
    n = min(step, n - part * step);
  }
  *begin = plain_load(row_starts + lo);
  *end = plain_load(row_starts + lo + 1);
  return *begin <= row && row < *end ? lo : -1;
}

// Two float32 operations in one instruction; each half is rounded like the single operation.
__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split_f32x2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// A block appends up to kAppendTokens rows.  hd / 16 lanes share a head: lane l holds the groups of eight entries at 8 l
// and hd/2 + 8 l, so the two halves that the rotary positions pair lie in one lane, and of the Hadamard rotation's stages
// only those at distances hd/4 to 8 need exchanges.  A warp takes 512 / hd query, key or value heads (one kind) through
// the block's rows, the next row's entries loaded while it works on this one's; where the rows go (sequence, position,
// page) is found once per block, by a warp per row, while the first entries are on their way; the same warp puts the
// position's angles into shared memory (read by every warp from global memory they cost 22 of 132 us).  What bounds many
// rows is the issue of instructions (79 % of the cycles, 424 a warp and 512 entries, 48 of them exchanges between lanes):
// 18.9k rows of 48 heads of 128 in 110 us, 4.5 TB/s.  Exchanges that swap halves between lanes need half as many
// shuffles, but the selections around them cost more: 119 us.
constexpr int kAppendMaxWarps = 12;
constexpr int kAppendTokens = 4;

struct TokenPlace {
  long long at;  // (page heads << page_shift) + offset in the page
  int pos;       // -1: the row is skipped
};

template <typename T>
struct Raw16;
template <>
struct Raw16<__nv_bfloat16> {
  uint4 v[2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int half) {
    v[0] = *reinterpret_cast<const uint4*>(p);
    v[1] = *reinterpret_cast<const uint4*>(p + half);
  }
  __device__ __forceinline__ void get(float (&y)[2][8]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      y[i][0] = bf16_lo(v[i].x); y[i][1] = bf16_hi(v[i].x); y[i][2] = bf16_lo(v[i].y); y[i][3] = bf16_hi(v[i].y);
      y[i][4] = bf16_lo(v[i].z); y[i][5] = bf16_hi(v[i].z); y[i][6] = bf16_lo(v[i].w); y[i][7] = bf16_hi(v[i].w);
    }
  }
};
template <>
struct Raw16<float> {
  float4 v[4];
  __device__ __forceinline__ void load(const float* p, int half) {
    v[0] = *reinterpret_cast<const float4*>(p);
    v[1] = *reinterpret_cast<const float4*>(p + 4);
    v[2] = *reinterpret_cast<const float4*>(p + half);
    v[3] = *reinterpret_cast<const float4*>(p + half + 4);
  }
  __device__ __forceinline__ void get(float (&y)[2][8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i / 2][i % 2 * 4] = v[i].x; y[i / 2][i % 2 * 4 + 1] = v[i].y;
      y[i / 2][i % 2 * 4 + 2] = v[i].z; y[i / 2][i % 2 * 4 + 3] = v[i].w;
    }
  }
};

// Rotary positions (entries i and i + hd/2 are a pair), then the normalised Hadamard rotation, stages from the widest to
// the narrowest: the order fixes the roundings.  All lanes of the warp take part.  angles: the row's, as stored by
// k_kv_append.
template <int HD>
__device__ __forceinline__ void turn_head(float (&y)[2][8], int sub, const float4* angles, bool hadamard,
                                          float had_scale) {
  constexpr int LPH = HD / 16;
  const uint64_t minus = f32x2(-1.f, -1.f);
  uint64_t z[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) z[i][e] = f32x2(y[i][2 * e], y[i][2 * e + 1]);
  if (angles != nullptr) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 f = angles[5 * sub + e];  // c, c, s, s
      // (products one by one: ptxas merges a paired product with a paired sum into one rounding)
      auto times = [](uint64_t v, float lo, float hi) {
        float a, b;
        split_f32x2(v, a, b);
        return f32x2(__fmul_rn(a, lo), __fmul_rn(b, hi));
      };
      const uint64_t a = z[0][e], b = z[1][e];
      z[0][e] = fma2(times(b, f.z, f.w), minus, times(a, f.x, f.y));
      z[1][e] = add2(times(b, f.x, f.y), times(a, f.z, f.w));
    }
  }
  if (hadamard) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // distance hd/2
      const uint64_t a = z[0][e], b = z[1][e];
      z[0][e] = add2(a, b);
      z[1][e] = fma2(b, minus, a);
    }
#pragma unroll
    for (int w = LPH / 2; w >= 1; w >>= 1) {  // distances 8 w: the other lane's entry plus or minus one's own
      const uint64_t sign = (sub & w) ? minus : f32x2(1.f, 1.f);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[i][e] = fma2(z[i][e], sign, __shfl_xor_sync(0xffffffffu, z[i][e], w));
    }
    const uint64_t scale2 = f32x2(had_scale, had_scale);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int w = 2; w >= 1; w >>= 1) {  // distances 2 w
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((e & w) == 0) {
            const uint64_t a = z[i][e], b = z[i][e + w];
            z[i][e] = add2(a, b);
            z[i][e + w] = fma2(b, minus, a);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // distance 1
        float a, b;
        split_f32x2(z[i][e], a, b);
        z[i][e] = mul2(f32x2(__fadd_rn(a, b), __fsub_rn(a, b)), scale2);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) split_f32x2(z[i][e], y[i][2 * e], y[i][2 * e + 1]);
}

// Range, step and codes of a head; stores codes, step and (if wanted) the values they stand for.
template <int HD, int BITS>
__device__ __forceinline__ void hold_head(const AppendParams& p, float (&y)[2][8], int sub, bool active,
                                          uint8_t* codes, float2* step, __nv_bfloat16* values) {
  constexpr int LPH = HD / 16;
  constexpr float kHalf = static_cast<float>(1 << (BITS - 1));
  float mn = y[0][0], mx = y[0][0];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mn = min_nan(mn, y[i][e]);
      mx = max_nan(mx, y[i][e]);
    }
  }
#pragma unroll
  for (int o = 1; o < LPH; o <<= 1) {
    mn = min_nan(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  if (!active) return;
  float scale, low = 0.f, shift;
  if (p.asym) {
    low = shift = __fmul_rn(mn, p.clip);
    scale = __fdiv_rn(__fsub_rn(__fmul_rn(mx, p.clip), low), p.den);
  } else {
    scale = __fdiv_rn(__fmul_rn(max_nan(mx, -mn), p.clip), p.den);
    shift = __fmul_rn(-scale, kHalf);
  }
  // an infinity or a NaN (or a range, or a shift, past float32): scale and shift NaN, codes 0
  if (!(scale < __uint_as_float(0x7f800000u)) || !(fabsf(shift) < __uint_as_float(0x7f800000u)))
    scale = shift = __uint_as_float(0x7fc00000u);
  const bool divide = quant_needs_division(scale), clamp = p.clip != 1.f;
  const float inv = divide ? 0.f : __frcp_rn(scale);
  const float lo = p.asym ? 0.f : -p.den, off = p.asym ? 0.f : kHalf;
  if (sub == 0) *step = make_float2(scale, shift);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float u[8];
    uint32_t w[8];
    if (scale > 0.f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] = __fsub_rn(y[i][e], low);
      quant8(y[i], scale, inv, divide, clamp, lo, p.den, off, u, w);
    } else {
      const float zero = scale == 0.f ? off : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = zero, w[e] = static_cast<uint32_t>(zero);
    }
    if constexpr (BITS == 4) {
      const uint32_t ev = pack_bytes(w[0], w[2], w[4], w[6]), od = pack_bytes(w[1], w[3], w[5], w[7]);
      *reinterpret_cast<uint32_t*>(codes + HD / 4 * i + 4 * sub) = (ev & 0x0f0f0f0fu) | ((od & 0x0f0f0f0fu) << 4);
    } else {
      *reinterpret_cast<uint2*>(codes + HD / 2 * i + 8 * sub) =
          make_uint2(pack_bytes(w[0], w[1], w[2], w[3]), pack_bytes(w[4], w[5], w[6], w[7]));
    }
    if (values != nullptr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = __fadd_rn(__fmul_rn(u[e], scale), shift);
      store8(values + HD / 2 * i, u);
    }
  }
}

template <typename T, int HD, int BITS, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, WARPS == 4 ? 6 : 2) k_kv_append(const AppendParams p) {
  constexpr int LPH = HD / 16;    // lanes per head
  constexpr int HPW = 32 / LPH;   // heads per warp
  constexpr int RB = HD * BITS / 8;
  __shared__ TokenPlace place[kAppendTokens];
  __shared__ float4 turns[kAppendTokens][LPH * 5];  // two pairs' c, c, s, s; a lane's four in a row, 80 bytes
                                                    // from lane to lane (no bank conflicts)
  wait_for_earlier_kernels();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const int sub = lane % LPH;
  const long long row0 = static_cast<long long>(blockIdx.x) * p.tokens;
  const int n_tok = static_cast<int>(min(static_cast<long long>(p.tokens), p.rows - row0));
  const int H = p.c.heads, Hq = p.q != nullptr ? p.q_heads : 0;
  const int uq = (Hq + HPW - 1) / HPW, uk = (H + HPW - 1) / HPW;  // units of heads of one kind

  // A unit is up to HPW heads of one kind; of a kind with fewer heads it takes as many rows at a time as there is room for
  // (45k rows of 2 query and 2 + 2 cache heads of 128: 60 us, a row at a time 93).
  int unit = warp;
  int head, off, per;  // the lane's head and its row among the `per` rows at a time
  bool active;
  long long step;      // elements from the lane's row to its next
  const T* src;
  auto source = [&](int u) {
    const T* base;
    int heads;
    long long ld;
    if (u < uq) base = static_cast<const T*>(p.q), ld = p.ldq, heads = Hq;
    else if (u < uq + uk) u -= uq, base = static_cast<const T*>(p.k), ld = p.ldk, heads = H;
    else u -= uq + uk, base = static_cast<const T*>(p.v), ld = p.ldv, heads = H;
    head = u * HPW + lane / LPH;
    off = 0;
    per = 1;
    if (heads < HPW) {
      per = HPW / heads;
      off = head / heads;
      head -= off * heads;
    }
    active = head < heads && off < per && off < n_tok;
    if (!active) head = 0, off = 0;  // (reads a real head, writes nothing)
    src = base + (row0 + off) * ld + head * HD + 8 * sub;
    step = ld * per;
  };
  Raw16<T> raw;
  source(unit);
  raw.load(src, HD / 2);

  for (int t = warp; t < n_tok; t += n_warps) {
    const int row = static_cast<int>(row0) + t;
    TokenPlace w;
    w.pos = -1;
    w.at = 0;
    float4 turn = make_float4(0.f, 0.f, 0.f, 0.f);
    int begin, end;
    const int s = find_sequence(p.b.row_starts, p.b.n_seqs, row, &begin, &end);
    unsigned int wrong = 0u;
    if (s >= 0) {
      const int length = plain_load(p.b.lengths + s);
      const int pos = max(length, 0) - (end - row);
      // (a sequence whose rows do not fit is skipped whole, as the attention does: its rows' positions cannot be told)
      if (begin < 0 || end > p.rows || end - begin > p.b.max_rows || length < 0 || pos < 0 || length > p.b.max_length ||
          static_cast<long long>(length) > (static_cast<long long>(p.b.table_ld) << p.c.page_shift) ||
          (p.rope != nullptr && pos >= p.rope_rows)) {
        wrong = kCacheErrBatch;
      } else {
        if (p.rope != nullptr && lane < LPH * 4)
          turn = plain_load(reinterpret_cast<const float4*>(p.rope + static_cast<long long>(pos) * HD) + lane);
        const int page =
            plain_load(p.b.page_table + static_cast<long long>(s) * p.b.table_ld + (pos >> p.c.page_shift));
        if (page < 0 || page >= p.c.pages) {
          wrong = kCacheErrPage;
        } else {
          w.pos = pos;
          w.at = (static_cast<long long>(page) * H << p.c.page_shift) + (pos & ((1 << p.c.page_shift) - 1));
        }
      }
    } else if (row >= plain_load(p.b.row_starts) && row < plain_load(p.b.row_starts + p.b.n_seqs)) {
      wrong = kCacheErrBatch;  // starts that do not ascend
    }
    if (wrong != 0u && lane == 0) atomicMax(p.err, wrong);
    if (lane == 0) place[t] = w;
    if (lane < LPH * 4) turns[t][lane / 4 * 5 + lane % 4] = make_float4(turn.x, turn.z, turn.y, turn.w);
  }
  __syncthreads();

  while (true) {
    for (int t = 0; t < n_tok;) {
      float y[2][8];
      raw.get(y);
      const int at_row = min(t + off, n_tok - 1), mine = unit, my_head = head;
      const long long row = row0 + at_row;
      const int pos = place[at_row].pos;
      const bool my_active = active && t + off < n_tok && pos >= 0;
      t += per;
      if (t < n_tok) {
        if (t + off < n_tok) src += step;  // (else the lane's last row once more, for nothing)
        raw.load(src, HD / 2);
      } else {
        unit += n_warps;
        if (unit < uq + 2 * uk) {
          source(unit);
          raw.load(src, HD / 2);
        }
      }
      if (!__any_sync(0xffffffffu, my_active)) continue;
      const float4* angles = p.rope != nullptr ? turns[at_row] : nullptr;
      if (mine < uq) {
        turn_head<HD>(y, sub, angles, p.hadamard, p.had_scale);
        if (my_active) {
          __nv_bfloat16* dst = p.q_out + row * p.ldqo + my_head * HD + 8 * sub;
          store8(dst, y[0]);
          store8(dst + HD / 2, y[1]);
        }
      } else {
        const bool is_k = mine < uq + uk;
        if (is_k) turn_head<HD>(y, sub, angles, p.hadamard, p.had_scale);
        const long long at = place[at_row].at + (static_cast<long long>(my_head) << p.c.page_shift);
        __nv_bfloat16* values = is_k ? p.k_values : p.v_values;
        if (values != nullptr) values += row * (is_k ? p.ldkv : p.ldvv) + my_head * HD + 8 * sub;
        hold_head<HD, BITS>(p, y, sub, my_active, (is_k ? p.c.k_codes : p.c.v_codes) + at * RB,
                            (is_k ? p.c.k_steps : p.c.v_steps) + at, values);
      }
    }
    if (unit >= uq + 2 * uk) break;
  }
}

}  // namespace kt
