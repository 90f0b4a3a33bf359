// Attention over the paged, quantised cache for few query rows per sequence (a decode step, a few tokens verified
// together).
//
// With u the code of an entry from zero upwards and (s, b) its token's scale and shift, key and value are s u + b, so
//   q.k_t          = s_t (q.u_t) + b_t sum(q)
//   sum_t p_t v_t  = sum_t (p_t s_t) u_t + sum_t p_t b_t
// and the codes themselves (centred on zero) are the operands of the tensor cores: small integers are exact in float16,
// so no rounding of the cache is added, and no entry is ever scaled.  float16 and not bf16, because its ten fraction bits
// take a 4-bit code from either half of a byte, or an 8-bit code, without a shift: turning codes into operands is most of
// this kernel's instructions (64 sequences of up to 8192 tokens, 4 bits: with bf16 the ALU pipe was 72 % busy, with float16
// it is 48 %, issue slots 60 %; no unit is full, and 16 warps an SM do not hide each other's latencies).  The other
// operands get a power of two that keeps them inside float16's range.  A query row: the one that brings its largest entry to
// 2^14.  Its bf16 entries are exact then down to 2^-31 of that power of two; with 4-bit codes the odd ones, which are held 16
// times smaller, down to 2^-27; smaller ones are off by 2^-39 (odd ones 2^-35) of it at most.  p_t s_t: the one that brings the
// row's largest p_t s_t so far to 2^2 (terms below 2^-16 of it are off by 2^-27 of it at most).  Rounding p_t s_t to float16,
// 2^-11 of itself at most, is the only other rounding before the output's; scores, softmax statistics, sums and outputs are
// float32.
//
// Layout of the work.  A row is a query head of one token; the rows of one key head (group x tokens) are packed into
// blocks of 8 NT.  All tiles of 32 tokens of all blocks form one list, cut into equal runs, one per CTA that the device
// holds at a time: sequences of any lengths leave no CTA with more than its share (chunks of a fixed length cost 100 to
// 130 us where this takes 80, by how they filled the last wave).  A CTA's run crosses blocks; where it covers a block
// whole it writes the output, else one of its two partial results (its first block's and its last one's), which a second
// kernel joins.  Within a run the warps take tiles in turn, each with its own maximum, sum and output, joined in shared
// memory.  The products are transposed (tokens x rows, dims x rows): 16 tokens by 8 rows is the instruction's shape, so a
// group of 8 heads or fewer wastes little, and the code words of a token's row go from shared memory to the operand
// registers without any exchange between lanes (the contraction's order over the entries is free as long as the query is
// packed alike).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "serve_cache.cuh"
#include "sm100_prims.cuh"

namespace kt {

struct AttendParams {
  CacheView c;
  BatchView b;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;          // null: not wanted
  long long ldq, ldo;  // lse is dense: [rows][q_heads]
  int rows;            // rows of q and out
  int q_heads, group;  // group = q_heads / heads
  int row_blocks;      // blocks of 8 NT rows per sequence and key head
  int chunks, chunk_tokens;  // (prompts)
  float scale_log2;    // softmax scale * log2(e)
  int causal, window;
  float* part_o;       // rows: [CTAs][2][8 NT][hd]; prompts: [items][8 NT][hd], null when chunks == 1
  float2* part_ml;     // the same without [hd]: maximum (log2 units), sum
  int2* spans;         // rows: [blocks] the CTAs that hold a block's parts, first and last; the first one's slot in bit 31
  unsigned int group_magic;  // ceil(2^32 / group), 0 for a group of one
  uint32_t k1024;      // rows: 0x64006400
  int seq0, seqs;      // the sequences of this launch: seq0 .. seq0 + seqs - 1
  unsigned int* err;
};

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
  const int n = valid ? 16 : 0;  // 0: the destination is filled with zeros, nothing is read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// float16 x float16 -> float32
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t bf16x2_sub(uint32_t a, uint32_t b) {
  __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
// Two 8-bit codes in bits 0-7 and 16-23 (the others are ignored) to bf16 code - 128, exactly: 128 + (u mod 128) minus
// 128 or 256, both bf16 bit patterns built from the code's bits.
__device__ __forceinline__ uint32_t codes8_to_bf16(uint32_t w) {
  const uint32_t a = (w & 0x007f007fu) | 0x43004300u;
  const uint32_t b = (~w & 0x00800080u) | 0x43004300u;
  return bf16x2_sub(a, b);
}
// Two 4-bit codes in bits 0-3 and 16-19 to bf16 128 + code.
__device__ __forceinline__ uint32_t codes4_to_bf16_128(uint32_t w) { return (w & 0x000f000fu) | 0x43004300u; }

__device__ __forceinline__ uint32_t h2_add(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Pairs of codes in bits 0-3 and 16-19 to float16 code - 8, in bits 4-7 and 20-23 to 16 (code - 8), in bits 0-7 and 16-23
// to code - 128 (all other bits are ignored): put into the fraction of 1024, then one exact addition.  (The factor 16 is
// taken out of the other operand, or of the output: undoing it here costs a second constant's register.)
// `k1024` is float16 1024 twice, from a register the compiler cannot see through: with both constants known it takes two
// instructions for the and-or.
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t k1024) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "n"(MASK), "r"(k1024));
  return r;
}
__device__ __forceinline__ uint32_t nibbles_lo(uint32_t w, uint32_t k1024) {
  return h2_add(and_or<0x000f000fu>(w, k1024), 0xe408e408u);  // - 1032
}
__device__ __forceinline__ uint32_t nibbles_hi16(uint32_t w, uint32_t k1024) {
  return h2_add(and_or<0x00f000f0u>(w, k1024), 0xe480e480u);  // - 1152
}
__device__ __forceinline__ uint32_t bytes_f16(uint32_t w, uint32_t k1024) {
  return h2_add(and_or<0x00ff00ffu>(w, k1024), 0xe480e480u);  // - 1152
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ int exponent(float x) { return (__float_as_int(x) >> 23) - 127; }  // x > 0
// 2^(2 - exponent(x))
__device__ __forceinline__ float held_up(float x) {
  return __uint_as_float((256u << 23) - (__float_as_uint(x) & 0x7f800000u));
}

// What a CTA's block of rows is, the same for the attention and for the join of its chunks.
struct BlockOfRows {
  int first_row;  // of the batch
  int n_rows;     // tokens of the sequence in the batch
  int length;
  int lo, hi;     // tokens that any row of the block sees: [lo, hi), lo a multiple of 32 (128 for blocks of 256 rows)
  int n_rows_packed;
};
// r / group.  The rows kernel's packed rows are at most 128: a product is exact, and short (its code runs once or twice).
template <int NR>
__device__ __forceinline__ int over_group(const AttendParams& p, int r) {
  if (NR > 16) return r / p.group;
  return p.group_magic == 0u ? r : static_cast<int>(__umulhi(static_cast<unsigned int>(r), p.group_magic));
}
template <int NR>
__device__ __forceinline__ bool block_of_rows(const AttendParams& p, int seq, int rb, BlockOfRows* o) {
  const int r0 = plain_load(p.b.row_starts + seq), r1 = plain_load(p.b.row_starts + seq + 1);
  int length = plain_load(p.b.lengths + seq);
  o->first_row = r0;
  o->n_rows = r1 - r0;
  const long long most = static_cast<long long>(p.b.table_ld) << p.c.page_shift;
  if (r0 < 0 || o->n_rows < 0 || r1 > p.rows || o->n_rows > p.b.max_rows || length < 0 || length > p.b.max_length || length > most) {
    atomicMax(p.err, kCacheErrBatch);
    return false;
  }
  o->length = length;
  o->n_rows_packed = o->n_rows * p.group;
  const int first = rb * NR;
  if (first >= o->n_rows_packed) return false;
  const int last = min(first + NR, o->n_rows_packed) - 1;
  const int past = length - o->n_rows;  // position of the first row (negative: rows that see nothing)
  const int pos_first = past + over_group<NR>(p, first), pos_last = past + over_group<NR>(p, last);
  o->hi = p.causal ? max(0, min(length, pos_last + 1)) : length;
  o->lo = p.window > 0 ? max(0, pos_first - p.window + 1) & ~(NR > 16 ? 127 : 31) : 0;
  o->lo = min(o->lo, o->hi);
  return true;
}

// Length of a block of rows in the list of all tiles: kBlockCost for taking it up (the query, the first tiles' latency,
// the join of the warps, in tiles), then its tiles (one where the rows see nothing, so that someone writes them); 0 if
// there is no such block.  Without that cost a run over many short sequences took twice as long as one over a long one.
constexpr int kBlockCost = 16;
template <int NR>
__device__ __forceinline__ int block_tiles(const AttendParams& p, int seq, int rb, BlockOfRows* blk) {
  if (!block_of_rows<NR>(p, seq, rb, blk)) return 0;
  return kBlockCost + max(1, (blk->hi - blk->lo + 31) >> 5);
}
template <int NR>
__device__ __forceinline__ long long sequence_tiles(const AttendParams& p, int seq) {  // of one key head
  long long n = 0;
  BlockOfRows blk;
  for (int rb = 0; rb < p.row_blocks; ++rb) n += block_tiles<NR>(p, seq, rb, &blk);
  return n;
}
// Tiles of a CTA's run: the list in as many equal runs as there are CTAs, one tile per warp at least.
__device__ __forceinline__ long long run_tiles(long long total, int ctas, int warps) {
  const long long n = total >> 31 == 0 ? (static_cast<unsigned int>(total) + ctas - 1u) / static_cast<unsigned int>(ctas)
                                       : (total + ctas - 1) / ctas;
  return n < warps ? warps : n;
}

template <int HD, int BITS, int NT, int WARPS, int STAGES>
struct AttendConfig {
  static constexpr int RB = HD * BITS / 8;
  static constexpr int kTile = 32;
  static constexpr int kStageBytes = 2 * kTile * RB + 2 * kTile * 8;
  static constexpr int kRing = WARPS * STAGES * kStageBytes;
  static constexpr int NR = 8 * NT;
  static constexpr int kJoin = WARPS * NR * (HD + 4) * 4;  // each warp's output rows, maximum and sum
  static constexpr int kSmem = kRing > kJoin ? kRing : kJoin;
};

template <int HD, int BITS, int NT, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32, NT == 1 ? 4 : 2) k_kv_attend_rows(const AttendParams p) {
  using Cfg = AttendConfig<HD, BITS, NT, WARPS, STAGES>;
  constexpr int RB = Cfg::RB, NR = Cfg::NR;
  constexpr int KS = HD / 16;        // contraction steps of the scores
  constexpr int MT = HD / 16;        // dimension tiles of the output
  constexpr int CPR = RB / 16;       // 16-byte pieces of a token's codes
  constexpr int WPL = HD / 4 * BITS / 32;   // code words a lane holds of a key row
  constexpr int VW = HD / 8 * BITS / 32;    // and of a value row
  extern __shared__ __align__(128) uint8_t smem[];
  wait_for_earlier_kernels();
  const uint32_t k1024 = p.k1024;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, c = lane & 3;

  // --- the CTA's run of the list of tiles.  Every warp adds up the sequences' tiles, 32 sequences at a time, and keeps
  // the sums in its part of the ring while they fit.
  constexpr int kSums = STAGES * Cfg::kStageBytes / 8;
  long long* sums = reinterpret_cast<long long*>(smem + warp * STAGES * Cfg::kStageBytes);
  auto scan = [&](int s0) {  // inclusive sums over 32 sequences
    long long n = s0 + lane < p.b.n_seqs ? sequence_tiles<NR>(p, s0 + lane) * p.c.heads : 0;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, n, x);
      if (lane >= x) n += up;
    }
    return n;
  };
  long long total = 0;
  for (int s0 = 0; s0 < p.b.n_seqs; s0 += 32) {
    const long long n = total + scan(s0);
    if (s0 + lane < min(p.b.n_seqs, kSums)) sums[s0 + lane] = n;
    total = __shfl_sync(0xffffffffu, n, 31);
  }
  const long long run = run_tiles(total, gridDim.x, WARPS);
  const long long run_begin = blockIdx.x * run, run_end = min(total, run_begin + run);
  if (run_begin >= run_end) return;
  __syncwarp();
  int seq = 0;
  long long before = 0;  // tiles in front of the sequence
  for (int s0 = 0;; s0 += 32) {
    const bool kept = p.b.n_seqs <= kSums;
    const long long n = !kept ? before + scan(s0) : s0 + lane < p.b.n_seqs ? sums[s0 + lane] : total;
    const unsigned int reach = __ballot_sync(0xffffffffu, n > run_begin);  // (the last sum is the total, which is)
    if (reach != 0u) {
      const int l = __ffs(reach) - 1;
      seq = s0 + l;
      if (l > 0) before = __shfl_sync(0xffffffffu, n, l - 1);
      break;
    }
    before = __shfl_sync(0xffffffffu, n, 31);
  }
  __syncthreads();  // (the ring is written from here on)
  long long per_head = sequence_tiles<NR>(p, seq);
  int head;
  long long skip;  // tiles of the head in front of the run, then of the block
  if (((run_begin - before) | per_head) >> 31 == 0) {
    head = static_cast<int>(static_cast<unsigned int>(run_begin - before) / static_cast<unsigned int>(per_head));
    skip = static_cast<unsigned int>(run_begin - before) - static_cast<unsigned int>(head) * static_cast<unsigned int>(per_head);
  } else {
    head = static_cast<int>((run_begin - before) / per_head);
    skip = (run_begin - before) % per_head;
  }
  int rb = 0;
  BlockOfRows blk;
  int in_block = block_tiles<NR>(p, seq, rb, &blk);
  while (skip >= in_block) {
    skip -= in_block;
    in_block = block_tiles<NR>(p, seq, ++rb, &blk);
  }

  for (long long pos = run_begin; pos < run_end;) {
  // --- one block, or the part of it that lies in the run
  const int seg = static_cast<int>(min(run_end - pos, static_cast<long long>(in_block) - skip));
  const int tile0 = max(0, static_cast<int>(skip) - kBlockCost), tile1 = static_cast<int>(skip) + seg - kBlockCost;
  if (tile1 <= 0) break;  // (the run ends before the block's first tile)
  const bool whole = tile0 == 0 && tile1 == in_block - kBlockCost;
  if (threadIdx.x == 0) {  // for the join
    int2* span = p.spans + (static_cast<long long>(seq) * p.c.heads + head) * p.row_blocks + rb;
    if (tile0 == 0) span->x = static_cast<int>(blockIdx.x) | (pos == run_begin ? 0 : 1 << 31);
    if (tile1 == in_block - kBlockCost) span->y = blockIdx.x;
  }
  const int t_begin = blk.lo + tile0 * 32;
  const int t_end = min(blk.hi, blk.lo + tile1 * 32);
  const int past = blk.length - blk.n_rows;
  const int first = rb * NR;

  // the query as the second operand: row n = g of every 8-row tile, entries paired like the codes of a key word
  uint32_t qf[NT][KS][2];
  float qsum[NT][2], down[NT][2];  // of the scaled query; the factor that undoes the scale, times scale log2(e)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = first + nt * 8 + g;
    uint32_t w[HD / 8];  // lane c's HD/4 entries
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) w[i] = 0u;
    if (r < blk.n_rows_packed) {
      const uint4* src = reinterpret_cast<const uint4*>(
          p.q + (blk.first_row + over_group<NR>(p, r)) * p.ldq +
          (head * p.group + r - over_group<NR>(p, r) * p.group) * HD + c * (HD / 4));
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        const uint4 v = plain_load(src + i);
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) top = max(top, max(w[i] << 16 & 0x7fff0000u, w[i] & 0x7fff0000u));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // (0 and what is no number: no factor)
    const int e = top == 0u || top >= 0x7f800000u ? 0 : min(126, 141 - static_cast<int>(top >> 23));
    const float up = power_of_two(e);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) {
      const float lo = bf16_lo(w[i]) * up, hi = bf16_hi(w[i]) * up;
      sum += lo + hi;
      w[i] = pack_f16(lo, BITS == 4 ? hi * 0.0625f : hi);  // (odd entries meet codes times 16)
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      qsum[nt][i] = __shfl_sync(0xffffffffu, sum, 8 * c + 4 * i);
      down[nt][i] = power_of_two(-__shfl_sync(0xffffffffu, e, 8 * c + 4 * i)) * p.scale_log2;
    }
    if constexpr (BITS == 4) {
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {  // eight entries, two steps: pairs (e, e + 4)
        qf[nt][2 * i][0] = __byte_perm(w[4 * i], w[4 * i + 2], 0x5410);
        qf[nt][2 * i][1] = __byte_perm(w[4 * i], w[4 * i + 2], 0x7632);
        qf[nt][2 * i + 1][0] = __byte_perm(w[4 * i + 1], w[4 * i + 3], 0x5410);
        qf[nt][2 * i + 1][1] = __byte_perm(w[4 * i + 1], w[4 * i + 3], 0x7632);
      }
    } else {
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {  // four entries, one step: pairs (e, e + 2)
        qf[nt][i][0] = __byte_perm(w[2 * i], w[2 * i + 1], 0x5410);
        qf[nt][i][1] = __byte_perm(w[2 * i], w[2 * i + 1], 0x7632);
      }
    }
  }
  // tokens that the lane's rows (columns 2c, 2c + 1 of every tile) see: [see_lo, see_hi)
  int see_lo[NT][2], see_hi[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = min(first + nt * 8 + 2 * c + i, blk.n_rows_packed - 1);
      const int pos = past + over_group<NR>(p, r);
      see_hi[nt][i] = p.causal ? min(blk.length, pos + 1) : blk.length;
      see_lo[nt][i] = p.window > 0 ? pos - p.window + 1 : 0;
    }
  }
  // every row of the block sees [all_lo, all_hi): tiles inside need no mask
  const int all_hi = p.causal ? min(blk.length, past + over_group<NR>(p, first) + 1) : blk.length;
  const int all_lo =
      p.window > 0 ? past + over_group<NR>(p, min(first + NR, blk.n_rows_packed) - 1) - p.window + 1 : 0;

  float o[NT][MT][4];
  float m[NT][2], l[NT][2], bs[NT][2];
  float big[NT][2];     // the largest p_t |s_t| of a row (2^-100 at least): its output is held times held_up(big)
  float limit = 0.f;    // a value scale from here on might pass float16's range in one of the lane's rows
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 2; ++i) m[nt][i] = -INFINITY, l[nt][i] = 0.f, bs[nt][i] = 0.f, big[nt][i] = power_of_two(-100);
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[nt][j][e] = 0.f;
  }

  // --- the warp's ring of tiles
  const int n_tiles = (t_end - t_begin + 31) >> 5;
  const uint32_t ring = smem_u32(smem) + warp * STAGES * Cfg::kStageBytes;
  const uint8_t* ring_ptr = smem + warp * STAGES * Cfg::kStageBytes;
  const int* table = p.b.page_table + static_cast<long long>(seq) * p.b.table_ld;
  const int page_mask = (1 << p.c.page_shift) - 1;
  const bool two_pages = p.c.page_shift == 4;  // pages of 16 tokens: a tile has two
  // page ids of the tile at t (the second half's beside it); -1 past the end
  auto page_ids = [&](int tile, int* a, int* b) {
    const int t = t_begin + tile * 32;
    *a = tile < n_tiles ? plain_load(table + (t >> p.c.page_shift)) : -1;
    *b = (two_pages && tile < n_tiles && t + 16 < t_end) ? plain_load(table + ((t + 16) >> 4)) : *a;
  };
  auto fetch = [&](int tile, int stage, int id0, int id1) {
    if (tile < n_tiles) {
      const int t0 = t_begin + tile * 32;
      const bool ok0 = id0 >= 0 && id0 < p.c.pages, ok1 = id1 >= 0 && id1 < p.c.pages;
      const long long base0 = (static_cast<long long>(ok0 ? id0 : 0) * p.c.heads + head) << p.c.page_shift;
      const uint32_t dst = ring + stage * Cfg::kStageBytes + lane * 16;
      if (!two_pages && ok0 && t0 + 32 <= t_end) {  // 32 tokens in a row
        const long long at = base0 + (t0 & page_mask);
        const uint8_t* ks = p.c.k_codes + at * RB + lane * 16;
        const uint8_t* vs = p.c.v_codes + at * RB + lane * 16;
#pragma unroll
        for (int i = 0; i < CPR; ++i) {
          cp_async16(dst + i * 512, ks + i * 512, true);
          cp_async16(dst + 32 * RB + i * 512, vs + i * 512, true);
        }
        cp_async16(dst + 64 * RB, (lane < 16 ? p.c.k_steps : p.c.v_steps) + at + (lane & 15) * 2, true);
      } else {
        if ((!ok0 || !ok1) && lane == 0) atomicMax(p.err, kCacheErrPage);
        const long long base1 = (static_cast<long long>(ok1 ? id1 : 0) * p.c.heads + head) << p.c.page_shift;
#pragma unroll
        for (int i = 0; i < CPR; ++i) {
          const int piece = i * 32 + lane, t = piece / CPR;
          const bool second = two_pages && t >= 16;
          const bool valid = t0 + t < t_end && (second ? ok1 : ok0);
          const long long at = ((second ? base1 : base0) + ((t0 + t) & page_mask)) * RB + (piece % CPR) * 16;
          cp_async16(dst + i * 512, p.c.k_codes + at, valid);
          cp_async16(dst + 32 * RB + i * 512, p.c.v_codes + at, valid);
        }
        // steps: 16 pieces of two tokens for the keys, 16 for the values
        const int t = (lane & 15) * 2;
        const bool second = two_pages && t >= 16;
        const long long at = (second ? base1 : base0) + ((t0 + t) & page_mask);
        cp_async16(dst + 64 * RB, (lane < 16 ? p.c.k_steps : p.c.v_steps) + at,
                   (second ? ok1 : ok0) && t0 + t < t_end);
      }
    }
    cp_async_commit();
  };
  int id0, id1;
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) {
    page_ids(warp + i * WARPS, &id0, &id1);
    fetch(warp + i * WARPS, i, id0, id1);
  }
  page_ids(warp + (STAGES - 1) * WARPS, &id0, &id1);

  int stage = 0;
  for (int tile = warp; tile < n_tiles; tile += WARPS) {
    {
      const int next = stage == 0 ? STAGES - 1 : stage - 1;
      fetch(tile + (STAGES - 1) * WARPS, next, id0, id1);
      page_ids(tile + STAGES * WARPS, &id0, &id1);
    }
    cp_async_wait<STAGES - 1>();
    __syncwarp();
    const uint8_t* st = ring_ptr + stage * Cfg::kStageBytes;
    const int t0 = t_begin + tile * 32;

    // scores of 32 tokens x 8 NT rows
    float s[NT][2][4];
    uint32_t wa[2][WPL], wb[2][WPL];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][mt][e] = 0.f;
      const uint8_t* ka = st + (mt * 16 + g) * RB + c * WPL * 4;
      const uint8_t* kb = ka + 8 * RB;
      if constexpr (WPL == 2) {
        const uint2 a = *reinterpret_cast<const uint2*>(ka), b = *reinterpret_cast<const uint2*>(kb);
        wa[mt][0] = a.x; wa[mt][1] = a.y; wb[mt][0] = b.x; wb[mt][1] = b.y;
      } else {
#pragma unroll
        for (int i = 0; i < WPL / 4; ++i) {
          const uint4 a = *reinterpret_cast<const uint4*>(ka + 16 * i), b = *reinterpret_cast<const uint4*>(kb + 16 * i);
          wa[mt][4 * i] = a.x; wa[mt][4 * i + 1] = a.y; wa[mt][4 * i + 2] = a.z; wa[mt][4 * i + 3] = a.w;
          wb[mt][4 * i] = b.x; wb[mt][4 * i + 1] = b.y; wb[mt][4 * i + 2] = b.z; wb[mt][4 * i + 3] = b.w;
        }
      }
    }
#pragma unroll
    for (int w = 0; w < WPL; ++w) {  // (the two tiles of 16 tokens in turn: two independent chains of products)
      if constexpr (BITS == 4) {
#pragma unroll
        for (int hstep = 0; hstep < 2; ++hstep) {
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            const uint32_t x = wa[mt][w] >> (8 * hstep), y = wb[mt][w] >> (8 * hstep);
            const uint32_t a[4] = {nibbles_lo(x, k1024), nibbles_lo(y, k1024), nibbles_hi16(x, k1024), nibbles_hi16(y, k1024)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_16816(s[nt][mt], a, qf[nt][2 * w + hstep][0], qf[nt][2 * w + hstep][1]);
          }
        }
      } else {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const uint32_t a[4] = {bytes_f16(wa[mt][w], k1024), bytes_f16(wb[mt][w], k1024), bytes_f16(wa[mt][w] >> 8, k1024),
                                 bytes_f16(wb[mt][w] >> 8, k1024)};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_16816(s[nt][mt], a, qf[nt][w][0], qf[nt][w][1]);
        }
      }
    }

    // s (q.c) + b sum(q) with c the centred codes and b their shift; times `down` it is the score in log2 units
    constexpr float kMid = BITS == 4 ? 8.f : 128.f;
    const float2* ksteps = reinterpret_cast<const float2*>(st + 64 * RB);
    const float2* vsteps = ksteps + 32;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float2 f = ksteps[mt * 16 + half * 8 + g];
        const float fb = fmaf(kMid, f.x, f.y);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            s[nt][mt][half * 2 + i] = fmaf(s[nt][mt][half * 2 + i], f.x, fb * qsum[nt][i]);
      }
    }
    const bool masked = t0 < all_lo || t0 + 32 > min(all_hi, t_end);
    if (masked) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int t = t0 + mt * 16 + half * 8 + g;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (t < see_lo[nt][i] || t >= see_hi[nt][i] || t >= t_end) s[nt][mt][half * 2 + i] = -INFINITY;
        }
    }
    // maximum per row: over the lane's four tokens, then over the eight lanes that share its rows.  The reference m that
    // the probabilities are taken against moves only when the maximum has passed it by more than 8 (a factor of 2^8):
    // moving it costs every output register a product.
    float mx[NT][2];
    bool moved = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float v = fmaxf(fmaxf(s[nt][0][i], s[nt][0][2 + i]), fmaxf(s[nt][1][i], s[nt][1][2 + i]));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
        mx[nt][i] = v * down[nt][i];
        moved |= mx[nt][i] > m[nt][i] + 8.f;
      }
    float2 vf[2][2];
    float vtop = 0.f;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        vf[mt][half] = vsteps[mt * 16 + half * 8 + g];
        vtop = fmaxf(vtop, fabsf(vf[mt][half].x));  // (NaN has no say)
      }
    if (masked || __any_sync(0xffffffffu, moved || vtop >= limit)) {
      limit = INFINITY;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float m_new = mx[nt][i] > m[nt][i] + 8.f ? mx[nt][i] : m[nt][i];
          // the largest p s among the tokens that the row sees, and of those before it, against the new reference
          float t = power_of_two(-100);
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const float y = s[nt][mt][half * 2 + i];
              if (y != -INFINITY) t = fmaxf(t, fabsf(exp2_fast(fmaf(y, down[nt][i], -m_new)) * vf[mt][half].x));
            }
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
          const int e_old = exponent(big[nt][i]);
          float back = 0.f, back_o = 0.f;  // what the sums and the output are multiplied with
          if (m[nt][i] != -INFINITY) {
            const float moves = m[nt][i] - m_new;
            // (a product with 2^moves could underflow where what it scales does not)
            t = fmaxf(t, moves == 0.f ? big[nt][i] : exp2_fast(moves + static_cast<float>(e_old + 1)));
            t = fminf(t, power_of_two(126));
            back = exp2_fast(moves);
            back_o = exp2_fast(moves + static_cast<float>(e_old - exponent(t)));
          }
          big[nt][i] = fminf(t, power_of_two(126));
          limit = fminf(limit, power_of_two(min(127, exponent(big[nt][i]) + 5)));
          m[nt][i] = m_new;
          l[nt][i] *= back;
          bs[nt][i] *= back;
          f[i] = back_o;
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          o[nt][j][0] *= f[0]; o[nt][j][1] *= f[1];
          o[nt][j][2] *= f[0]; o[nt][j][3] *= f[1];
        }
      }
    }
    // probabilities, and the second product's operand p_t s_t (held_up, below 2^15 as p < 2^8, rounded to float16)
    // transposed to tokens x rows
    uint32_t pf[NT][2][2];
    auto probabilities = [&](auto hidden) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float fb = fmaf(kMid, vf[mt][half].x, vf[mt][half].y);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float y = s[nt][mt][half * 2 + i];
              float pr = exp2_fast(fmaf(y, down[nt][i], -m[nt][i]));
              const bool none = decltype(hidden)::value && y == -INFINITY;
              if (none) pr = 0.f;
              l[nt][i] += pr;
              bs[nt][i] += none ? 0.f : pr * fb;  // (not 0 times what a hidden token may hold)
              // (p first: s times the power of two may pass float32's range where p is 0)
              w[i] = none ? 0.f : pr * vf[mt][half].x * held_up(big[nt][i]);
            }
            pf[nt][mt][half] = transpose8x8(pack_f16(w[0], w[1]));
          }
        }
    };
    if (masked) probabilities(std::true_type{});
    else probabilities(std::false_type{});
    // outputs: dims x rows
    const uint8_t* vst = st + 32 * RB;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      uint32_t w[4][VW];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int t = mt * 16 + 2 * c + (k & 1) + (k >> 1) * 8;
        const uint8_t* src = vst + t * RB + g * VW * 4;
        if constexpr (VW == 1) {
          w[k][0] = *reinterpret_cast<const uint32_t*>(src);
        } else if constexpr (VW == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(src);
          w[k][0] = v.x; w[k][1] = v.y;
        } else {
          const uint4 v = *reinterpret_cast<const uint4*>(src);
          w[k][0] = v.x; w[k][1] = v.y; w[k][2] = v.z; w[k][3] = v.w;
        }
      }
#pragma unroll
      for (int i = 0; i < VW; ++i) {
#pragma unroll
        for (int hw = 0; hw < 2; ++hw) {
          const uint32_t ab = __byte_perm(w[0][i], w[1][i], hw ? 0x7632 : 0x5410);
          const uint32_t cd = __byte_perm(w[2][i], w[3][i], hw ? 0x7632 : 0x5410);
          if constexpr (BITS == 4) {  // four entries: two dimension tiles
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              const uint32_t x = ab >> (8 * jj), y = cd >> (8 * jj);
              const uint32_t a[4] = {nibbles_lo(x, k1024), nibbles_hi16(x, k1024), nibbles_lo(y, k1024), nibbles_hi16(y, k1024)};
              const int j = i * 4 + hw * 2 + jj;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_16816(o[nt][j], a, pf[nt][mt][0], pf[nt][mt][1]);
            }
          } else {  // two entries: one dimension tile
            const uint32_t a[4] = {bytes_f16(ab, k1024), bytes_f16(ab >> 8, k1024), bytes_f16(cd, k1024), bytes_f16(cd >> 8, k1024)};
            const int j = i * 2 + hw;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_16816(o[nt][j], a, pf[nt][mt][0], pf[nt][mt][1]);
          }
        }
      }
    }
    __syncwarp();
    stage = stage == STAGES - 1 ? 0 : stage + 1;
  }
  cp_async_wait<0>();
  __syncthreads();

  // --- join the warps.  o[nt][j][0..1]: dim g HD/8 + 2j, rows 2c, 2c + 1; [2..3]: the next dim
  float* join = reinterpret_cast<float*>(smem);
  constexpr int kRow = HD + 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float ll = l[nt][i], bb = bs[nt][i];
#pragma unroll
      for (int x = 4; x <= 16; x <<= 1) {
        ll += __shfl_xor_sync(0xffffffffu, ll, x);
        bb += __shfl_xor_sync(0xffffffffu, bb, x);
      }
      // A value that is no number makes the row's sum NaN, which every join keeps: its output would be lost where this part
      // lies so far below the row's maximum that its factor is 0.
      if (!(fabsf(bb) < __uint_as_float(0x7f800000u))) ll = __uint_as_float(0x7fc00000u);
      float* dst = join + (warp * NR + nt * 8 + 2 * c + i) * kRow;
      const float g_down = power_of_two(exponent(big[nt][i]) - 2);
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        dst[g * (HD / 8) + 2 * j] = fmaf(o[nt][j][i], g_down, bb);
        dst[g * (HD / 8) + 2 * j + 1] = fmaf(o[nt][j][2 + i], BITS == 4 ? g_down * 0.0625f : g_down, bb);
      }
      if (g == 0) {
        dst[HD] = m[nt][i];
        dst[HD + 1] = ll;
      }
    }
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < NR * (HD / 4); idx += WARPS * 32) {
    const int r = idx / (HD / 4), e = idx % (HD / 4) * 4;
    if (first + r >= blk.n_rows_packed) continue;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, join[(w * NR + r) * kRow + HD]);
    float sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float* src = join + (w * NR + r) * kRow;
      const float f = src[HD] == -INFINITY && src[HD + 1] == 0.f ? 0.f : exp2_fast(src[HD] - top);
      const float4 v = *reinterpret_cast<const float4*>(src + e);
      sum = fmaf(f, src[HD + 1], sum);
      if (f != 0.f) {
        acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y);
        acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
      }
    }
    if (whole) {
      const int pr = first + r;
      const int in_seq = over_group<NR>(p, pr);
      const long long row = blk.first_row + in_seq;
      const int qh = head * p.group + pr - in_seq * p.group;
      const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;  // a row that sees nothing: zeros
      uint2 v;
      v.x = pack_bf16(acc.x * inv, acc.y * inv);
      v.y = pack_bf16(acc.z * inv, acc.w * inv);
      *reinterpret_cast<uint2*>(p.out + row * p.ldo + qh * HD + e) = v;
      if (p.lse != nullptr && e == 0)
        p.lse[row * p.q_heads + qh] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    } else {
      const long long at = (blockIdx.x * 2ll + (pos == run_begin ? 0 : 1)) * NR + r;
      *reinterpret_cast<float4*>(p.part_o + at * HD + e) = acc;
      if (e == 0) p.part_ml[at] = make_float2(top, sum);
    }
  }
  // --- the next block
  pos += seg;
  if (pos < run_end) {
    skip = 0;
    in_block = ++rb < p.row_blocks ? block_tiles<NR>(p, seq, rb, &blk) : 0;
    if (in_block == 0) {
      rb = 0;
      if (++head >= p.c.heads) {
        head = 0;
        do {
          in_block = block_tiles<NR>(p, ++seq, 0, &blk);
        } while (in_block == 0);
      } else {
        in_block = block_tiles<NR>(p, seq, 0, &blk);
      }
    }
    __syncthreads();  // (the ring's memory held the join)
  }
  }
}

// Joins the parts of the blocks that several CTAs worked on, in the order of the runs: one CTA per block, a warp per row, or
// (SPREAD) one CTA per row, whose warps take a range of the parts each and are joined in that order.
template <int HD, int NT, bool SPREAD>
__global__ void __launch_bounds__(256) k_kv_attend_join_runs(const AttendParams p) {
  constexpr int NR = 8 * NT;
  __shared__ float ranges[SPREAD ? 8 : 1][HD + 2];
  wait_for_earlier_kernels();
  const int lane = threadIdx.x & 31;
  const int warp = threadIdx.x >> 5;
  unsigned int item = SPREAD ? blockIdx.x / NR : blockIdx.x;
  const int2 span = p.spans[item];
  const int rb = static_cast<int>(item % p.row_blocks);
  item /= p.row_blocks;
  const int head = static_cast<int>(item % p.c.heads);
  const int seq = static_cast<int>(item / p.c.heads);
  BlockOfRows blk;
  if (!block_of_rows<NR>(p, seq, rb, &blk)) return;
  const int c0 = span.x & 0x7fffffff, c1 = span.y;
  if (c0 == c1) return;  // written whole
  const int first_slot = span.x < 0 ? 1 : 0;
  const int each = (c1 - c0 + 8) / 8;
  const int a = SPREAD ? c0 + warp * each : c0, b = SPREAD ? min(c1, a + each - 1) : c1;
  for (int r = SPREAD ? blockIdx.x % NR : warp; r < NR; r += SPREAD ? NR : 8) {
    const int pr = rb * NR + r;
    if (pr >= blk.n_rows_packed) break;
    auto part = [&](int c) { return (c * 2ll + (c == c0 ? first_slot : 0)) * NR + r; };
    float top = -INFINITY, sum = 0.f;
    float acc[HD / 32];
#pragma unroll
    for (int e = 0; e < HD / 32; ++e) acc[e] = 0.f;
    for (int base = a; base <= b; base += 32) {
      const float2 ml = base + lane <= b ? p.part_ml[part(base + lane)] : make_float2(-INFINITY, 0.f);
      const bool none = ml.x == -INFINITY && ml.y == 0.f;
      float t = none ? -INFINITY : ml.x;
#pragma unroll
      for (int x = 16; x >= 1; x >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
      t = fmaxf(t, top);
      const float old = top == -INFINITY ? 0.f : exp2_fast(top - t);
      const float f = none ? 0.f : exp2_fast(ml.x - t);
      float part_sum = none ? 0.f : ml.y * f;
#pragma unroll
      for (int x = 16; x >= 1; x >>= 1) part_sum += __shfl_xor_sync(0xffffffffu, part_sum, x);
      sum = sum * old + part_sum;
      top = t;
#pragma unroll
      for (int e = 0; e < HD / 32; ++e) acc[e] *= old;
      const int n = min(32, b - base + 1);
#pragma unroll 8
      for (int k = 0; k < n; ++k) {
        const float fk = __shfl_sync(0xffffffffu, f, k);
        const float* src = p.part_o + part(base + k) * HD + lane * (HD / 32);
        float v[HD / 32];
        if constexpr (HD == 128) {
          const float4 q = *reinterpret_cast<const float4*>(src);
          v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
        } else {
          const float2 q = *reinterpret_cast<const float2*>(src);
          v[0] = q.x, v[1] = q.y;
        }
#pragma unroll
        for (int e = 0; e < HD / 32; ++e) acc[e] = fk == 0.f ? acc[e] : fmaf(fk, v[e], acc[e]);
      }
    }
    if constexpr (SPREAD) {
#pragma unroll
      for (int e = 0; e < HD / 32; ++e) ranges[warp][lane * (HD / 32) + e] = acc[e];
      if (lane == 0) ranges[warp][HD] = top, ranges[warp][HD + 1] = sum;
      __syncthreads();  // (all warps of the CTA have the same row)
      if (warp != 0) return;
      float most = -INFINITY;
#pragma unroll
      for (int w = 0; w < 8; ++w) most = fmaxf(most, ranges[w][HD]);
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < HD / 32; ++e) acc[e] = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const float t = ranges[w][HD], l = ranges[w][HD + 1];
        const float f = t == -INFINITY && l == 0.f ? 0.f : exp2_fast(t - most);
        sum = fmaf(f, l, sum);  // (the factor 0 too: a range may hold NaN only, or far below the others)
        if (f == 0.f) continue;
#pragma unroll
        for (int e = 0; e < HD / 32; ++e) acc[e] = fmaf(f, ranges[w][lane * (HD / 32) + e], acc[e]);
      }
      top = most;
    }
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const int in_seq = over_group<NR>(p, pr);
    const long long row = blk.first_row + in_seq;
    const int qh = head * p.group + pr - in_seq * p.group;
    __nv_bfloat16* dst = p.out + row * p.ldo + qh * HD + lane * (HD / 32);
    if constexpr (HD == 128)
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    else
      *reinterpret_cast<uint32_t*>(dst) = pack_bf16(acc[0] * inv, acc[1] * inv);
    if (p.lse != nullptr && lane == 0)
      p.lse[row * p.q_heads + qh] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
  }
}

// Joins the chunks of every row: one warp per packed row of a block, in the order of the chunks.
template <int HD, int NT>
__global__ void __launch_bounds__(128) k_kv_attend_join(const AttendParams p) {
  constexpr int NR = 8 * NT, E = HD / 32;
  const int lane = threadIdx.x & 31;
  long long item = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  const int r = static_cast<int>(item % NR);
  item /= NR;
  const long long block = item;
  const int rb = static_cast<int>(item % p.row_blocks);
  item /= p.row_blocks;
  const int head = static_cast<int>(item % p.c.heads);
  const int seq = p.seq0 + static_cast<int>(item / p.c.heads);
  if (seq >= p.seq0 + p.seqs) return;
  BlockOfRows blk;
  if (!block_of_rows<NR>(p, seq, rb, &blk)) return;
  const int pr = rb * NR + r;
  if (pr >= blk.n_rows_packed) return;
  const int chunks = min(p.chunks, max(1, (blk.hi - blk.lo + p.chunk_tokens - 1) / p.chunk_tokens));
  float top = -INFINITY, sum = 0.f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int k = 0; k < chunks; ++k) {
    const long long at = (block * p.chunks + k) * NR + r;
    const float2 ml = p.part_ml[at];
    const float* src = p.part_o + at * HD + lane * E;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = src[e];
    if (ml.x == -INFINITY && ml.y == 0.f) continue;
    const float t = fmaxf(top, ml.x);
    const float fo = top == -INFINITY ? 0.f : exp2_fast(top - t), fn = exp2_fast(ml.x - t);
    sum = sum * fo + ml.y * fn;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = acc[e] * fo + v[e] * fn;
    top = t;
  }
  const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
  const long long row = blk.first_row + pr / p.group;
  const int qh = head * p.group + pr % p.group;
  __nv_bfloat16* dst = p.out + row * p.ldo + qh * HD + lane * E;
#pragma unroll
  for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t*>(dst + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
  if (p.lse != nullptr && lane == 0)
    p.lse[row * p.q_heads + qh] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

}  // namespace kt
