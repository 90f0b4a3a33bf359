// Launch side of the serving operators: argument checks, the choice of a kernel's shape, scratch layout.
#include "serve.h"

#include <math.h>

#include <mutex>

#include "serve_attend.cuh"
#include "serve_cache.cuh"
#include "serve_norm.cuh"
#include "serve_prompt.cuh"
#include "sm100_prims.cuh"

namespace kt {

#define SV_CUDA(call)              \
  do {                             \
    if ((call) != cudaSuccess) {   \
      (void)cudaGetLastError();    \
      return KT_ERR_CUDA;          \
    }                              \
  } while (0)
#define SV_TRY(expr)                \
  do {                              \
    kt_status st__ = (expr);        \
    if (st__ != KT_OK) return st__; \
  } while (0)

static kt_status launched(ServeCtx* sc) {
  SV_CUDA(cudaGetLastError());
  ++sc->launches;
  return KT_OK;
}
static bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static int element_bytes(int dtype) { return dtype == KT_BF16 ? 2 : 4; }

// Opt-in to `bytes` of dynamic shared memory, once per kernel and device (devices beyond the table: every launch).
constexpr int kMaxDevices = 64;
struct SmemOptIn {
  bool done[kMaxDevices];
};
static std::mutex g_optin_mutex;
template <typename K>
static kt_status opt_in(SmemOptIn* o, K kernel, int device, int bytes) {
  std::lock_guard<std::mutex> lock(g_optin_mutex);
  if (device < kMaxDevices && o->done[device]) return KT_OK;
  SV_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (device < kMaxDevices) o->done[device] = true;
  return KT_OK;
}

// CTAs of a kernel that an SM holds, `most` at most; asked for once per kernel and device.
struct Residency {
  int held[kMaxDevices];
};
template <typename K>
static kt_status resident(Residency* r, K kernel, int device, int threads, int bytes, int most, int* per_sm) {
  std::lock_guard<std::mutex> lock(g_optin_mutex);
  *per_sm = device < kMaxDevices ? r->held[device] : 0;
  if (*per_sm > 0) return KT_OK;
  SV_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(per_sm, kernel, threads, bytes));
  if (*per_sm < 1) return KT_ERR_CUDA;
  if (*per_sm > most) *per_sm = most;
  if (device < kMaxDevices) r->held[device] = *per_sm;
  return KT_OK;
}

// ------------------------------------------------------------------------------------------------ RMSNorm
static kt_status check_rows(const kt_mat& m, int64_t rows, int64_t cols) {
  if (m.data == nullptr && rows > 0) return KT_ERR_INVALID_ARG;
  if (m.rows != rows || m.cols != cols || m.ld < cols) return KT_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(m.data) % element_bytes(m.dtype)) != 0) return KT_ERR_ALIGN;
  return KT_OK;
}

// A launch whose blocks may be placed while the stream's last kernel still runs; they wait for it (griddepcontrol.wait)
// before they read what it writes.
template <typename K, typename P>
static kt_status launch_early(ServeCtx* sc, K kernel, dim3 blocks, unsigned threads, size_t smem, const P& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = blocks;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = sc->stream;
  cudaLaunchAttribute early = {};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  SV_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
  return launched(sc);
}

template <typename T, int V, bool VEC, int LANES>
static kt_status launch_norm(ServeCtx* sc, const NormParams& p, int threads) {
  const int per_block = LANES > 0 ? threads / (LANES > 0 ? LANES : 1) : 1;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(p.rows) + per_block - 1) / per_block);
  return launch_early(sc, k_rmsnorm_quant<T, V, VEC, LANES>, blocks, threads, 0, p);
}

template <typename T, bool VEC>
static kt_status norm_shape(ServeCtx* sc, const NormParams& p) {
  const int groups = (p.d + (p.ahead ? 14 : 7)) / 8;  // groups of eight entries, one or more per thread
  // Rows of up to 128 entries share a warp (400000 rows of 128 71 us, a warp each 133).
  if (groups <= 8) return launch_norm<T, 1, VEC, 8>(sc, p, 128);
  if (groups <= 16) return launch_norm<T, 1, VEC, 16>(sc, p, 128);
  if (groups <= 32) return launch_norm<T, 1, VEC, 32>(sc, p, 128);
  if (groups <= 64) return launch_norm<T, 2, VEC, 32>(sc, p, 128);
  if (groups <= 128) return launch_norm<T, 4, VEC, 32>(sc, p, 128);
  auto threads = [&](int v) { return ((groups + v - 1) / v + 31) / 32 * 32; };
  // Two groups a thread where there are fewer rows than fill the device (a row's latency counts: 3.0 against 4.2 us for
  // one row of 4096, 5.7 against 7.1 for 257 of 8192), else four: blocks half as wide, more rows in flight on an SM
  // (16384 rows of 4096 with residual 113 against 122 us, 4099 of 14336 in float32 74 against 118).
  if (groups <= 2 * 1024 && p.rows <= 2 * sc->sm_count) return launch_norm<T, 2, VEC, 0>(sc, p, threads(2));
  return launch_norm<T, 4, VEC, 0>(sc, p, threads(4));
}

kt_status serve_rmsnorm_quant(ServeCtx* sc, const kt_mat& X, const kt_mat* residual, const kt_mat* sum,
                              const float* gain, double eps, const kt_quant_spec* spec, int8_t* codes, float* scales,
                              const kt_mat* values) {
  if (X.dtype != KT_BF16 && X.dtype != KT_F32) return KT_ERR_INVALID_ARG;
  if (X.rows < 0 || X.rows > 0x7fffffffll || X.cols < 1 || X.cols > 32768) return KT_ERR_SHAPE;
  SV_TRY(check_rows(X, X.rows, X.cols));
  if (sum != nullptr && residual == nullptr) return KT_ERR_INVALID_ARG;
  for (const kt_mat* m : {residual, sum}) {
    if (m == nullptr) continue;
    if (m->dtype != X.dtype) return KT_ERR_INVALID_ARG;
    SV_TRY(check_rows(*m, X.rows, X.cols));
  }
  if (!(eps >= 0.0) || !isfinite(eps)) return KT_ERR_INVALID_ARG;
  if (gain != nullptr && (reinterpret_cast<uintptr_t>(gain) & 3u) != 0) return KT_ERR_ALIGN;
  NormParams p = {};
  if (spec != nullptr) {
    if (spec->bits < 2 || spec->bits > 8 || spec->asymmetric != 0 || spec->clip_mode != 0 ||
        !(spec->clip > 0.f && spec->clip <= 1.f))
      return KT_ERR_INVALID_ARG;
    if (X.rows > 0 && (scales == nullptr || (codes == nullptr && values == nullptr))) return KT_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(scales) & 3u) != 0) return KT_ERR_ALIGN;
    p.bits = spec->bits;
    p.clip = spec->clip;
    p.den = static_cast<float>((1 << (spec->bits - 1)) - 1);
  } else if (codes != nullptr || scales != nullptr || values == nullptr) {
    return KT_ERR_INVALID_ARG;
  }
  if (values != nullptr) {
    if (values->dtype != KT_BF16 && values->dtype != KT_F32) return KT_ERR_INVALID_ARG;
    SV_TRY(check_rows(*values, X.rows, X.cols));
  }
  if (X.rows == 0) return KT_OK;
  p.x = X.data;
  p.ldx = X.ld;
  if (residual != nullptr) p.res = residual->data, p.ldr = residual->ld;
  if (sum != nullptr) p.sum = const_cast<void*>(sum->data), p.lds = sum->ld;
  if (values != nullptr) {
    p.values = const_cast<void*>(values->data);
    p.ldv = values->ld;
    p.values_f32 = values->dtype == KT_F32;
  }
  p.gain = gain;
  p.codes = codes;
  p.scales = scales;
  p.rows = static_cast<int>(X.rows);
  p.d = static_cast<int>(X.cols);
  p.eps = eps;
  bool vec = p.d % 8 == 0 && (reinterpret_cast<uintptr_t>(codes) & 7u) == 0;
  for (const kt_mat* m : {&X, residual, sum, values})
    if (m != nullptr) vec = vec && at16(m->data) && (m->ld * element_bytes(m->dtype)) % 16 == 0;
  p.ahead = !vec && p.d <= 32768 - 8;  // (one group more than d / 8 has to fit)
  if (X.dtype == KT_BF16) return vec ? norm_shape<__nv_bfloat16, true>(sc, p) : norm_shape<__nv_bfloat16, false>(sc, p);
  return vec ? norm_shape<float, true>(sc, p) : norm_shape<float, false>(sc, p);
}

// ------------------------------------------------------------------------------------------------ cache and batch
static kt_status check_cache(const kt_kv_cache& c, CacheView* v) {
  if (c.k_codes == nullptr || c.v_codes == nullptr || c.k_steps == nullptr || c.v_steps == nullptr)
    return KT_ERR_INVALID_ARG;
  if (c.bits != 4 && c.bits != 8) return KT_ERR_INVALID_ARG;
  if (c.head_dim != 64 && c.head_dim != 128) return KT_ERR_SHAPE;
  int shift = 4;
  while (shift < 8 && (1 << shift) != c.page_size) ++shift;
  if ((1 << shift) != c.page_size || c.pages < 1 || c.heads < 1) return KT_ERR_SHAPE;
  if (!at16(c.k_codes) || !at16(c.v_codes) || !at16(c.k_steps) || !at16(c.v_steps)) return KT_ERR_ALIGN;
  if (v != nullptr) {
    v->k_codes = static_cast<uint8_t*>(c.k_codes);
    v->v_codes = static_cast<uint8_t*>(c.v_codes);
    v->k_steps = reinterpret_cast<float2*>(c.k_steps);
    v->v_steps = reinterpret_cast<float2*>(c.v_steps);
    v->pages = c.pages;
    v->heads = c.heads;
    v->page_shift = shift;
  }
  return KT_OK;
}

static kt_status check_batch(const kt_kv_batch& b, BatchView* v) {
  if (b.row_starts == nullptr || b.lengths == nullptr || b.page_table == nullptr) return KT_ERR_INVALID_ARG;
  if (b.n_seqs < 1 || b.table_ld < 1 || b.max_rows < 0 || b.max_rows > (1 << 30) || b.max_length < 0 ||
      b.max_length > (1 << 30))
    return KT_ERR_SHAPE;
  for (const int32_t* i : {b.row_starts, b.lengths, b.page_table})
    if ((reinterpret_cast<uintptr_t>(i) & 3u) != 0) return KT_ERR_ALIGN;
  if (v != nullptr) {
    v->row_starts = b.row_starts;
    v->lengths = b.lengths;
    v->page_table = b.page_table;
    v->n_seqs = b.n_seqs;
    v->table_ld = b.table_ld;
    v->max_rows = b.max_rows;
    v->max_length = b.max_length;
  }
  return KT_OK;
}

// a matrix of heads: 16-byte aligned rows of `cols` elements
static kt_status check_heads(const kt_mat& m, int64_t rows, int64_t cols) {
  SV_TRY(check_rows(m, rows, cols));
  if (!at16(m.data) || (m.ld * element_bytes(m.dtype)) % 16 != 0) return KT_ERR_ALIGN;
  return KT_OK;
}

// ------------------------------------------------------------------------------------------------ append
template <typename T, int WARPS>
static kt_status launch_append(ServeCtx* sc, const AppendParams& p, int head_dim, int bits) {
  const unsigned blocks = static_cast<unsigned>((p.rows + p.tokens - 1) / p.tokens);
  const int per_warp = 512 / head_dim;  // heads a warp takes at a time
  const int units = ((p.q != nullptr ? p.q_heads : 0) + per_warp - 1) / per_warp + 2 * ((p.c.heads + per_warp - 1) / per_warp);
  const int rounds = (units + WARPS - 1) / WARPS;
  const int threads = (units + rounds - 1) / rounds * 32;
  if (head_dim == 128)
    return launch_early(sc, bits == 4 ? k_kv_append<T, 128, 4, WARPS> : k_kv_append<T, 128, 8, WARPS>, blocks, threads, 0, p);
  return launch_early(sc, bits == 4 ? k_kv_append<T, 64, 4, WARPS> : k_kv_append<T, 64, 8, WARPS>, blocks, threads, 0, p);
}

kt_status serve_kv_append(ServeCtx* sc, const kt_kv_cache& cache, const kt_kv_batch& batch, const kt_mat* Q,
                          const kt_mat& K, const kt_mat& V, const float* rope, int64_t rope_rows, int32_t hadamard,
                          const kt_quant_spec& spec, const kt_mat* Q_out, const kt_mat* K_values,
                          const kt_mat* V_values) {
  AppendParams p = {};
  SV_TRY(check_cache(cache, &p.c));
  SV_TRY(check_batch(batch, &p.b));
  if (spec.bits != cache.bits || (spec.asymmetric != 0 && spec.asymmetric != 1) || spec.clip_mode != 0 ||
      !(spec.clip > 0.f && spec.clip <= 1.f) || (hadamard != 0 && hadamard != 1))
    return KT_ERR_INVALID_ARG;
  if (K.dtype != KT_BF16 && K.dtype != KT_F32) return KT_ERR_INVALID_ARG;
  if (V.dtype != K.dtype || (Q != nullptr && Q->dtype != K.dtype)) return KT_ERR_INVALID_ARG;
  if ((Q == nullptr) != (Q_out == nullptr)) return KT_ERR_INVALID_ARG;
  const int64_t rows = K.rows, kv_cols = static_cast<int64_t>(cache.heads) * cache.head_dim;
  if (rows < 0 || rows > 0x7fffffffll) return KT_ERR_SHAPE;
  SV_TRY(check_heads(K, rows, kv_cols));
  SV_TRY(check_heads(V, rows, kv_cols));
  if (Q != nullptr) {
    if (Q->cols < cache.head_dim || Q->cols % cache.head_dim != 0 || Q->cols > 0x3fffffff) return KT_ERR_SHAPE;
    SV_TRY(check_heads(*Q, rows, Q->cols));
    if (Q_out->dtype != KT_BF16) return KT_ERR_INVALID_ARG;
    SV_TRY(check_heads(*Q_out, rows, Q->cols));
  }
  for (const kt_mat* m : {K_values, V_values}) {
    if (m == nullptr) continue;
    if (m->dtype != KT_BF16) return KT_ERR_INVALID_ARG;
    SV_TRY(check_heads(*m, rows, kv_cols));
  }
  if (rope != nullptr) {
    if (rope_rows < 1 || rope_rows > 0x7fffffffll) return KT_ERR_SHAPE;
    if (!at16(rope)) return KT_ERR_ALIGN;
  }
  if (rows == 0) return KT_OK;
  p.k = K.data, p.ldk = K.ld;
  p.v = V.data, p.ldv = V.ld;
  if (Q != nullptr) {
    p.q = Q->data, p.ldq = Q->ld;
    p.q_out = static_cast<__nv_bfloat16*>(const_cast<void*>(Q_out->data)), p.ldqo = Q_out->ld;
    p.q_heads = static_cast<int>(Q->cols / cache.head_dim);
  }
  if (K_values != nullptr)
    p.k_values = static_cast<__nv_bfloat16*>(const_cast<void*>(K_values->data)), p.ldkv = K_values->ld;
  if (V_values != nullptr)
    p.v_values = static_cast<__nv_bfloat16*>(const_cast<void*>(V_values->data)), p.ldvv = V_values->ld;
  p.rope = rope;
  p.rope_rows = static_cast<int>(rope_rows);
  p.rows = static_cast<int>(rows);
  p.hadamard = hadamard;
  p.asym = spec.asymmetric;
  p.clip = spec.clip;
  p.den = static_cast<float>(spec.asymmetric ? (1 << spec.bits) - 1 : (1 << (spec.bits - 1)) - 1);
  p.had_scale = static_cast<float>(1.0 / sqrt(static_cast<double>(cache.head_dim)));
  p.err = sc->cache_err;
  // several rows a block once blocks of one row would be many times what the device holds (4.. blocks an SM)
  const int64_t per_block = rows / (16ll * sc->sm_count);
  p.tokens = static_cast<int>(per_block < 1 ? 1 : per_block > kAppendTokens ? kAppendTokens : per_block);
  // Wide blocks where rows are fewer than the SMs' places (a row's latency counts: 64 rows 3.8 us with up to 12 warps,
  // 4.5 with 4), narrow ones else (18.9k rows of 48 heads of 128 110 us with 4, 137 with 12).
  if (rows <= 2ll * sc->sm_count)
    return K.dtype == KT_BF16 ? launch_append<__nv_bfloat16, kAppendMaxWarps>(sc, p, cache.head_dim, cache.bits)
                              : launch_append<float, kAppendMaxWarps>(sc, p, cache.head_dim, cache.bits);
  return K.dtype == KT_BF16 ? launch_append<__nv_bfloat16, 4>(sc, p, cache.head_dim, cache.bits)
                            : launch_append<float, 4>(sc, p, cache.head_dim, cache.bits);
}

// ------------------------------------------------------------------------------------------------ attention
constexpr int kRowWarps = 4, kRowStages = 3;
constexpr int kRowCtas = 4;  // CTAs an SM is given runs for, where it holds as many

// Rows of a key head from which the tensor-memory kernel is used.  Its tile is 256 rows, it reads what a first kernel has
// unpacked, and its smallest run is two tiles of tokens; the rows kernel reads and converts the cache once per 16 rows.  At
// 128 rows the two meet (rows against tiles, 8 key heads of 128, 4 bits: one sequence of 32768 tokens 97 and 98 us, of 8192
// 37 and 41, of 500 18 and 21, four of 8192 101 and 94), the rows kernel behind where there are many tokens (16 sequences of
// 2000 115 and 89, one of 131072 in 8 bits 524 and 339); at 64 it is far ahead (32768 tokens 54 and 97 us), at 256 behind
// (184 and 103).
constexpr long long kPromptRows = 129;
// Unpacked tiles held at a time; longer batches go in groups of sequences (one at least).
constexpr size_t kTileBudget = 1ull << 30;

struct AttendPlan {
  bool prompt;
  int nt, row_blocks, chunks, chunk_tokens;
  long long blocks;  // sequences (of a group) x key heads x row blocks
  int seqs;          // sequences of a group
  int tiles_per_seq;
  int ctas;          // rows: runs the list of tiles is cut into
  size_t tiles, part_ml, spans, total;  // partial outputs lie at `tiles` behind the unpacked tiles, then part_ml
};

static kt_status plan_attend(int sm_count, const kt_kv_cache& c, const kt_kv_batch& b, int q_heads, AttendPlan* pl) {
  *pl = AttendPlan{};
  const int group = q_heads / c.heads;
  const long long packed = static_cast<long long>(b.max_rows) * group;
  pl->prompt = packed >= kPromptRows;
  pl->nt = pl->prompt ? 32 : packed <= 8 ? 1 : 2;
  const int nr = 8 * pl->nt;
  const long long row_blocks = (packed + nr - 1) / nr;
  if (row_blocks * nr > 0x7fffffffll) return KT_ERR_SHAPE;  // (a block's first packed row is a 32-bit number)
  pl->row_blocks = static_cast<int>(row_blocks);
  pl->seqs = b.n_seqs;
  if (pl->prompt) {
    if (c.heads > 65535) return KT_ERR_SHAPE;
    pl->tiles_per_seq = (b.max_length + kTileTokens - 1) / kTileTokens;
    const size_t tile = c.head_dim == 128 ? PromptTile<128>::kBytes : PromptTile<64>::kBytes;
    const size_t per_seq = static_cast<size_t>(c.heads) * pl->tiles_per_seq * tile;
    const size_t fit = per_seq > 0 ? kTileBudget / per_seq : 65535;
    pl->seqs = static_cast<int>(fit < 1 ? 1 : fit > 65535 ? 65535 : fit);
    if (pl->seqs > b.n_seqs) pl->seqs = b.n_seqs;
    pl->tiles = (per_seq * pl->seqs + 255) / 256 * 256;
  }
  if (row_blocks > 0 && static_cast<long long>(pl->seqs) * c.heads > 0x7fffffffll / row_blocks) return KT_ERR_SHAPE;
  pl->blocks = static_cast<long long>(pl->seqs) * c.heads * row_blocks;
  if (!pl->prompt) {
    pl->ctas = kRowCtas * sm_count;
    const size_t rows = static_cast<size_t>(pl->ctas) * 2 * nr;
    pl->part_ml = rows * c.head_dim * 4;
    pl->spans = pl->part_ml + rows * 8;
    pl->total = pl->spans + static_cast<size_t>(pl->blocks) * 8;
    return KT_OK;
  }
  // Chunks of the tokens, one CTA an SM and at least two tiles each: as many as make the rounds of CTAs over the SMs cost
  // least, in steps of one tile.  A CTA's start and end cost five steps, the join two and a fortieth for every CTA's part
  // (168 blocks of 112 tiles: two rounds of whole blocks 498 us, four chunks a block 414; 64 blocks of 64 tiles: chunks of
  // 28, 28 and 8 tiles 120 us, two of 32 101; 8 blocks of 15 tiles: fours 29 us, twos 27).
  const long long tiles = pl->tiles_per_seq > 0 ? pl->tiles_per_seq : 1;
  long long best = 0, chunk = 0;
  for (long long n = 1; n == 1 || ((tiles + n - 1) / n >= 2 && n <= 64); ++n) {
    const long long each = (tiles + n - 1) / n, ctas = pl->blocks * n;
    const long long cost = 40 * ((ctas + sm_count - 1) / sm_count) * (each + 5) + (n > 1 ? 80 + ctas : 0);
    if (n == 1 || cost < best) best = cost, chunk = each * kTileTokens;
  }
  pl->chunk_tokens = static_cast<int>(chunk);
  pl->chunks = static_cast<int>((b.max_length + chunk - 1) / chunk);
  if (pl->chunks < 1) pl->chunks = 1;
  const long long items = pl->blocks * pl->chunks;
  if (items > 0x7fffffffll) return KT_ERR_SHAPE;
  pl->part_ml = pl->total = pl->tiles;
  if (pl->chunks > 1) {
    pl->part_ml = pl->tiles + (static_cast<size_t>(items) * nr * c.head_dim * 4 + 255) / 256 * 256;
    pl->total = pl->part_ml + static_cast<size_t>(items) * nr * 8;
  }
  return KT_OK;
}

kt_status serve_kv_scratch_bytes(int sm_count, const kt_kv_cache& cache, const kt_kv_batch& batch, int32_t q_heads,
                                 size_t* bytes) {
  SV_TRY(check_cache(cache, nullptr));
  SV_TRY(check_batch(batch, nullptr));
  if (q_heads < 1 || q_heads % cache.heads != 0) return KT_ERR_SHAPE;
  AttendPlan pl;
  SV_TRY(plan_attend(sm_count, cache, batch, q_heads, &pl));
  *bytes = pl.total;
  return KT_OK;
}

template <int HD, int NT>
static kt_status launch_join(ServeCtx* sc, const AttendParams& p, const AttendPlan& pl) {
  if (p.part_o == nullptr) return KT_OK;
  const long long warps = pl.blocks * 8 * NT;
  if ((warps + 3) / 4 > 0x7fffffffll) return KT_ERR_SHAPE;
  k_kv_attend_join<HD, NT><<<static_cast<unsigned>((warps + 3) / 4), 128, 0, sc->stream>>>(p);
  return launched(sc);
}

template <int HD, int BITS, int NT>
static kt_status launch_rows(ServeCtx* sc, const AttendParams& p, const AttendPlan& pl) {
  using Cfg = AttendConfig<HD, BITS, NT, kRowWarps, kRowStages>;
  static SmemOptIn optin;
  static Residency residency;
  auto kernel = k_kv_attend_rows<HD, BITS, NT, kRowWarps, kRowStages>;
  SV_TRY(opt_in(&optin, kernel, sc->device, Cfg::kSmem));
  int per_sm;
  SV_TRY(resident(&residency, kernel, sc->device, kRowWarps * 32, Cfg::kSmem, kRowCtas, &per_sm));
  const int ctas = per_sm * sc->sm_count;
  SV_TRY(launch_early(sc, kernel, ctas, kRowWarps * 32, Cfg::kSmem, p));
  // A CTA a row while those are few: their blocks may have hundreds of parts each (8 query heads on one key head over 131072
  // tokens: the call takes 26 us, 54 with a warp a row; 32 heads on 8 over 1500 tokens 9.5 and 10.6 us).
  if (pl.blocks * 8 * NT <= 8ll * sc->sm_count)
    return launch_early(sc, k_kv_attend_join_runs<HD, NT, true>, static_cast<unsigned>(pl.blocks * 8 * NT), 256, 0, p);
  return launch_early(sc, k_kv_attend_join_runs<HD, NT, false>, static_cast<unsigned>(pl.blocks), 256, 0, p);
}

template <int HD, int BITS>
static kt_status launch_prompt(ServeCtx* sc, const AttendParams& a, const AttendPlan& pl, void* scratch) {
  static SmemOptIn optin;
  auto kernel = k_kv_attend_tiles<HD>;
  SV_TRY(opt_in(&optin, kernel, sc->device, PromptSmem<HD>::kTotal));
  PromptParams p = {};
  p.a = a;
  p.tiles = static_cast<uint8_t*>(scratch);
  p.tiles_per_seq = pl.tiles_per_seq;
  p.err_word = sc->err_word;
  p.wait_limit_ns = sc->wait_limit_ns;
  for (int s = 0; s < a.b.n_seqs; s += pl.seqs) {
    p.a.seq0 = s;
    p.a.seqs = a.b.n_seqs - s < pl.seqs ? a.b.n_seqs - s : pl.seqs;
    // (launched even without tiles: the attention's blocks start early, behind it and all that came before it)
    const int tiles = pl.tiles_per_seq > 0 ? pl.tiles_per_seq : 1;
    SV_TRY(launch_early(sc, k_kv_unpack<HD, BITS>, dim3(tiles, a.c.heads, p.a.seqs), 256, 0, p));
    const long long items = static_cast<long long>(p.a.seqs) * a.c.heads * pl.row_blocks * pl.chunks;
    SV_TRY(launch_early(sc, kernel, static_cast<unsigned>(items), kPromptThreads, PromptSmem<HD>::kTotal, p));
    SV_TRY((launch_join<HD, 32>(sc, p.a, pl)));
  }
  return KT_OK;
}

template <int HD, int BITS>
static kt_status launch_attend(ServeCtx* sc, const AttendParams& p, const AttendPlan& pl, void* scratch) {
  if (pl.prompt) return launch_prompt<HD, BITS>(sc, p, pl, scratch);
  return pl.nt == 1 ? launch_rows<HD, BITS, 1>(sc, p, pl) : launch_rows<HD, BITS, 2>(sc, p, pl);
}

kt_status serve_kv_attend(ServeCtx* sc, const kt_kv_cache& cache, const kt_kv_batch& batch, const kt_mat& Q,
                          const kt_mat& out, float* lse, float scale, int32_t causal, int32_t window, void* scratch,
                          size_t scratch_bytes) {
  AttendParams p = {};
  SV_TRY(check_cache(cache, &p.c));
  SV_TRY(check_batch(batch, &p.b));
  if (Q.dtype != KT_BF16 || out.dtype != KT_BF16 || !(scale >= 0.f && scale <= 1e30f) || (causal != 0 && causal != 1) || window < 0)
    return KT_ERR_INVALID_ARG;
  if (Q.rows < 0 || Q.rows > 0x7fffffffll || Q.cols < 1 || Q.cols > 0x3fffffff ||
      Q.cols % (static_cast<int64_t>(cache.heads) * cache.head_dim) != 0)
    return KT_ERR_SHAPE;
  SV_TRY(check_heads(Q, Q.rows, Q.cols));
  SV_TRY(check_heads(out, Q.rows, Q.cols));
  const int q_heads = static_cast<int>(Q.cols / cache.head_dim);
  AttendPlan pl;
  SV_TRY(plan_attend(sc->sm_count, cache, batch, q_heads, &pl));
  if (pl.total > 0 && (scratch == nullptr || scratch_bytes < pl.total)) return KT_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(scratch) & 255u) != 0 || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0)
    return KT_ERR_ALIGN;
  if (Q.rows == 0 || pl.blocks == 0) return KT_OK;
  p.q = static_cast<const __nv_bfloat16*>(Q.data), p.ldq = Q.ld;
  p.out = static_cast<__nv_bfloat16*>(const_cast<void*>(out.data)), p.ldo = out.ld;
  p.lse = lse;
  p.rows = static_cast<int>(Q.rows);
  p.q_heads = q_heads;
  p.group = q_heads / cache.heads;
  p.group_magic = p.group == 1 ? 0u : static_cast<unsigned int>(((1ull << 32) + p.group - 1) / p.group);
  p.row_blocks = pl.row_blocks;
  p.chunks = pl.chunks;
  p.chunk_tokens = pl.chunk_tokens;
  p.scale_log2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  p.causal = causal;
  p.window = window < batch.max_length ? window : 0;  // (a wider one hides nothing; sums with it stay in 32 bits)
  p.err = sc->cache_err;
  p.seqs = batch.n_seqs;
  p.k1024 = 0x64006400u;
  if (pl.chunks > 1 || !pl.prompt) {
    p.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + pl.tiles);
    p.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(scratch) + pl.part_ml);
    p.spans = reinterpret_cast<int2*>(static_cast<uint8_t*>(scratch) + pl.spans);
  }
  if (cache.head_dim == 128)
    return cache.bits == 4 ? launch_attend<128, 4>(sc, p, pl, scratch) : launch_attend<128, 8>(sc, p, pl, scratch);
  return cache.bits == 4 ? launch_attend<64, 4>(sc, p, pl, scratch) : launch_attend<64, 8>(sc, p, pl, scratch);
}

}  // namespace kt
