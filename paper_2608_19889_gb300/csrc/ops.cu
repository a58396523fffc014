// C entry points of the operators on a paged key/value cache: attention that
// reads it, new tokens, and its blocks' management; and of tokens from logits. They check what the
// host can see, take the caller's buffers and launch; nothing is allocated and nothing is kept.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/axon.h"
#include "kernels.h"

namespace {

constexpr int MAX_ROWS = 8192;         // rows of a block table
constexpr int SAMPLE_MAX_ROWS = 1 << 24;
constexpr int MAX_BLOCKS_PER_SEQ = 1 << 26;  // positions fit 31 bits

bool unaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int check_cache(const axon_kv_cache* c) {
  if (!c || !c->k_pool || !c->v_pool || unaligned(c->k_pool) || unaligned(c->v_pool)) return AXON_ERR_INVALID_ARG;
  if (c->num_layers < 1 || c->num_blocks < 1 || c->num_kv_heads < 1) return AXON_ERR_INVALID_ARG;
  if (c->precision != AXON_BF16 && c->precision != AXON_FP16 && c->precision != AXON_FP32_DEBUG)
    return AXON_ERR_INVALID_ARG;
  if (c->block_size != 16 || (c->head_dim != 64 && c->head_dim != 128)) return AXON_ERR_UNSUPPORTED;
  return AXON_OK;
}

long long block_bytes(const axon_kv_cache* c) {
  return 16ll * c->num_kv_heads * c->head_dim * (c->precision == AXON_FP32_DEBUG ? 4 : 2);
}

// One layer's keys or values of a cache.
void* layer_pool(const axon_kv_cache* c, void* pool, int layer) {
  return static_cast<char*>(pool) + static_cast<long long>(layer) * c->num_blocks * block_bytes(c);
}

// The kernels' shared-memory limits belong to the device's context; they are set with the first
// attention call on a device, and again after its context was torn down (the launch of a kernel
// without them fails, and is then repeated once by with_limits).
template <typename Launch>
cudaError_t with_limits(Launch launch) {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  for (int round = 0; round < 2; ++round) {
    const bool known = (ready.load(std::memory_order_acquire) & bit) != 0;
    if (!known) {
      e = prepare_attn_chunk_kernels();
      if (e == cudaSuccess) e = prepare_attn_paged_kernels();
      if (e == cudaSuccess) e = prepare_attn_shared_kernels();
      if (e == cudaSuccess) e = prepare_sample_kernels();
      if (e != cudaSuccess) return e;
      ready.fetch_or(bit, std::memory_order_release);
    }
    e = launch();
    if (e != cudaErrorInvalidValue || !known) return e;
    cudaGetLastError();
    ready.fetch_and(~bit, std::memory_order_release);
  }
  return e;
}

int launch_ctx(const axon_kv_cache* c, void* stream, LaunchCtx* lc) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return AXON_ERR_CUDA;
  }
  *lc = LaunchCtx{static_cast<cudaStream_t>(stream), true, sms, c && c->precision == AXON_FP16};
  return AXON_OK;
}

int status(cudaError_t e) {
  if (e == cudaSuccess) return AXON_OK;
  cudaGetLastError();
  return AXON_ERR_CUDA;
}

// Strides of [rows][heads][head_dim] operands: 16-byte pieces, heads apart; a stride
// that nothing uses (one row, one head) is replaced by the dense one.
int check_strides(int rows, int heads, int d, int64_t& row, int64_t& head) {
  if (heads == 1) head = d;
  if (rows == 1) row = static_cast<int64_t>(heads) * (head > 0 ? head : d);
  if (row < d || head < d || row % 8 || head % 8 || row > (1ll << 36) || head > (1ll << 36)) return AXON_ERR_INVALID_ARG;
  return AXON_OK;
}

int check_attn(const axon_kv_cache* c, int layer, const void* q, const void* out, int num_heads, int blocks_per_seq,
               int window, int sinks, float scale) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (layer < 0 || layer >= c->num_layers || !q || !out || unaligned(q) || unaligned(out)) return AXON_ERR_INVALID_ARG;
  if (num_heads < 1 || num_heads % c->num_kv_heads || blocks_per_seq < 1 || blocks_per_seq > MAX_BLOCKS_PER_SEQ)
    return AXON_ERR_INVALID_ARG;
  if (window < 0 || sinks < 0 || !(scale >= 0.f) || isinf(scale)) return AXON_ERR_INVALID_ARG;
  if (c->precision == AXON_FP32_DEBUG || num_heads / c->num_kv_heads > 16) return AXON_ERR_UNSUPPORTED;
  return AXON_OK;
}

// Sinks that a row of `blocks` blocks can have (kernels round them up to blocks).
int clamp_sinks(int sinks, int blocks) {
  const int most = blocks * 16;  // blocks <= MAX_BLOCKS_PER_SEQ
  return sinks < most ? sinks : most;
}

float scale_log2(float scale, int d) {
  const double s = scale > 0.f ? static_cast<double>(scale) : 1.0 / sqrt(static_cast<double>(d));
  return static_cast<float>(s * 1.4426950408889634);
}

int pages_args(const axon_kv_cache* c, const axon_kv_seqs* s, void* work, int64_t work_bytes, int32_t* err,
               PagesArgs* a) {
  int rc = check_cache(c);
  if (rc) return rc;
  memset(a, 0, sizeof(*a));
  a->k = c->k_pool;
  a->v = c->v_pool;
  a->L = c->num_layers;
  a->N = c->num_blocks;
  a->block_bytes = block_bytes(c);
  a->err = err;
  if (!s) return AXON_OK;
  if (!s->block_table || !s->context_lens || !s->refs || s->max_seqs < 1 || s->blocks_per_seq < 1)
    return AXON_ERR_INVALID_ARG;
  if (s->max_seqs > MAX_ROWS || s->blocks_per_seq > MAX_BLOCKS_PER_SEQ ||
      static_cast<long long>(s->max_seqs) * s->blocks_per_seq > INT_MAX)
    return AXON_ERR_UNSUPPORTED;
  a->table = s->block_table;
  a->ctx = s->context_lens;
  a->refs = s->refs;
  a->R = s->max_seqs;
  a->P = s->blocks_per_seq;
  if (work_bytes >= 0) {
    if (!work || unaligned(work) ||
        static_cast<size_t>(work_bytes) < 4 * pages_work_ints(c->num_blocks, s->max_seqs, s->blocks_per_seq))
      return AXON_ERR_INVALID_ARG;
    a->work = static_cast<int*>(work);
  }
  return AXON_OK;
}

}  // namespace

namespace {

// Bytes of axon_attn_decode's part of a workspace.
size_t decode_bytes(const axon_kv_cache* c, int H, int sms) {
  return paged_attn_ticket_bytes(sms) + paged_attn_part_bytes(H, c->num_kv_heads, c->head_dim, sms);
}

// What the one-token forms have in common: checks and arguments, but for the workspace.
int decode_args(const axon_kv_cache* cache, int layer, const void* d_q, int64_t q_row_stride, int64_t q_head_stride, int B,
                int num_heads, const int32_t* d_context_lens, const int32_t* d_block_table, int blocks_per_seq, int window,
                int sinks, float scale, void* d_out, int64_t out_row_stride, int64_t out_head_stride, float* d_lse,
                void* d_workspace, int32_t* d_err, void* stream, LaunchCtx* lc, PagedAttnArgs* out) {
  int rc = check_attn(cache, layer, d_q, d_out, num_heads, blocks_per_seq, window, sinks, scale);
  if (rc) return rc;
  if (!d_context_lens || !d_workspace || unaligned(d_workspace) || B < 1) return AXON_ERR_INVALID_ARG;
  if (B > PAGED_ATTN_MAX_B || paged_attn_most_pages(B, cache->num_kv_heads, blocks_per_seq, window, sinks) > INT_MAX)
    return AXON_ERR_UNSUPPORTED;
  if ((rc = check_strides(B, num_heads, cache->head_dim, q_row_stride, q_head_stride)) ||
      (rc = check_strides(B, num_heads, cache->head_dim, out_row_stride, out_head_stride)))
    return rc;
  if (!d_block_table && static_cast<long long>(B) * blocks_per_seq > cache->num_blocks) return AXON_ERR_INVALID_ARG;
  if ((rc = launch_ctx(cache, stream, lc))) return rc;
  PagedAttnArgs& a = *out;
  memset(&a, 0, sizeof(a));
  a.q = d_q;
  a.q_row = q_row_stride;
  a.q_head = q_head_stride;
  a.k = layer_pool(cache, cache->k_pool, layer);
  a.v = layer_pool(cache, cache->v_pool, layer);
  a.ctx = d_context_lens;
  a.block_table = d_block_table;
  a.blocks_per_seq = blocks_per_seq;
  a.num_blocks = cache->num_blocks;
  a.B = B;
  a.H = num_heads;
  a.G = cache->num_kv_heads;
  a.d = cache->head_dim;
  a.window = window;
  a.sinks = window > 0 ? clamp_sinks(sinks, blocks_per_seq) : 0;
  a.scale_log2 = scale_log2(scale, cache->head_dim);
  a.o = d_out;
  a.o_row = out_row_stride;
  a.o_head = out_head_stride;
  a.lse = d_lse;
  a.ticket = static_cast<int*>(d_workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(d_workspace) + paged_attn_ticket_bytes(lc->num_sms));
  a.err = d_err;
  return AXON_OK;
}

}  // namespace

extern "C" {

int axon_attn_decode_workspace(const axon_kv_cache* cache, int32_t num_heads, int32_t B, int64_t* bytes) {
  int rc = check_cache(cache);
  if (rc) return rc;
  if (!bytes || num_heads < 1 || num_heads % cache->num_kv_heads || B < 1) return AXON_ERR_INVALID_ARG;
  if (num_heads / cache->num_kv_heads > 16 || B > PAGED_ATTN_MAX_B) return AXON_ERR_UNSUPPORTED;
  LaunchCtx lc;
  if ((rc = launch_ctx(cache, nullptr, &lc))) return rc;
  *bytes = static_cast<int64_t>(decode_bytes(cache, num_heads, lc.num_sms));
  return AXON_OK;
}

int axon_attn_decode(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride,
                     int64_t q_head_stride, int32_t B, int32_t num_heads, const int32_t* d_context_lens,
                     const int32_t* d_block_table, int32_t blocks_per_seq, int32_t window, int32_t sinks, float scale,
                     void* d_out, int64_t out_row_stride, int64_t out_head_stride, float* d_lse, void* d_workspace,
                     int64_t workspace_bytes, int32_t* d_err, void* stream) {
  LaunchCtx lc;
  PagedAttnArgs a;
  const int rc = decode_args(cache, layer, d_q, q_row_stride, q_head_stride, B, num_heads, d_context_lens, d_block_table,
                             blocks_per_seq, window, sinks, scale, d_out, out_row_stride, out_head_stride, d_lse, d_workspace,
                             d_err, stream, &lc, &a);
  if (rc) return rc;
  if (workspace_bytes < static_cast<int64_t>(decode_bytes(cache, num_heads, lc.num_sms))) return AXON_ERR_INVALID_ARG;
  return status(with_limits([&] { return launch_attn_paged_decode(lc, a); }));
}

int axon_attn_shared_workspace(const axon_kv_cache* cache, int32_t num_heads, int32_t B, int64_t* bytes) {
  int64_t own = 0;
  int rc = axon_attn_decode_workspace(cache, num_heads, B, bytes ? &own : nullptr);
  if (rc) return rc;
  LaunchCtx lc;
  if ((rc = launch_ctx(cache, nullptr, &lc))) return rc;
  *bytes = own + static_cast<int64_t>(shared_attn_bytes(B, num_heads, cache->head_dim, lc.num_sms));
  return AXON_OK;
}

int axon_attn_shared(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride, int64_t q_head_stride,
                     int32_t B, int32_t num_heads, const int32_t* d_context_lens, const int32_t* d_block_table,
                     int32_t blocks_per_seq, const int32_t* d_group_offsets, const int32_t* d_prefix_lens, int32_t num_groups,
                     int32_t window, int32_t sinks, float scale, void* d_out, int64_t out_row_stride, int64_t out_head_stride,
                     float* d_lse, void* d_workspace, int64_t workspace_bytes, int32_t* d_err, void* stream) {
  if (!d_block_table || !d_group_offsets || !d_prefix_lens || num_groups < 1) return AXON_ERR_INVALID_ARG;
  if (num_groups > SHARED_MAX_GROUPS) return AXON_ERR_UNSUPPORTED;
  LaunchCtx lc;
  PagedAttnArgs a;
  const int rc = decode_args(cache, layer, d_q, q_row_stride, q_head_stride, B, num_heads, d_context_lens, d_block_table,
                             blocks_per_seq, window, sinks, scale, d_out, out_row_stride, out_head_stride, d_lse, d_workspace,
                             d_err, stream, &lc, &a);
  if (rc) return rc;
  const size_t own = decode_bytes(cache, num_heads, lc.num_sms);
  if (workspace_bytes < static_cast<int64_t>(own + shared_attn_bytes(B, num_heads, a.d, lc.num_sms))) return AXON_ERR_INVALID_ARG;
  AttnMaps maps;
  if (!make_attn_maps_strided(&maps, d_q, B, a.q_row, a.q_head, a.k, a.v, static_cast<long long>(cache->num_blocks) * a.G * 16,
                              num_heads, a.G, a.d, lc.f16))
    return AXON_ERR_UNSUPPORTED;
  SharedGroups s;
  memset(&s, 0, sizeof(s));
  s.offsets = d_group_offsets;
  s.prefix = d_prefix_lens;
  s.N = num_groups;
  shared_attn_rules(&s, a, lc.num_sms);
  shared_attn_carve(&s, static_cast<char*>(d_workspace) + own, B, num_heads, a.d, lc.num_sms);
  return status(with_limits([&] { return launch_attn_shared(lc, a, s, maps); }));
}

int axon_attn_prefill(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride,
                      int64_t q_head_stride, int32_t B, int32_t T, int32_t num_heads, const int32_t* d_cu_seqlens,
                      const int32_t* d_context_lens, int32_t max_chunk, const int32_t* d_block_table,
                      int32_t blocks_per_seq, int32_t window, int32_t sinks, float scale, void* d_out,
                      int64_t out_row_stride, int64_t out_head_stride, int32_t* d_err, void* stream) {
  int rc = check_attn(cache, layer, d_q, d_out, num_heads, blocks_per_seq, window, sinks, scale);
  if (rc) return rc;
  if (!d_cu_seqlens || !d_context_lens || B < 1 || T < 1 || max_chunk < 1 || max_chunk > T) return AXON_ERR_INVALID_ARG;
  if ((rc = check_strides(T, num_heads, cache->head_dim, q_row_stride, q_head_stride)) ||
      (rc = check_strides(T, num_heads, cache->head_dim, out_row_stride, out_head_stride)))
    return rc;
  if (!d_block_table && static_cast<long long>(B) * blocks_per_seq > cache->num_blocks) return AXON_ERR_INVALID_ARG;
  if (static_cast<long long>(B) + T > INT_MAX / cache->num_kv_heads) return AXON_ERR_UNSUPPORTED;
  LaunchCtx lc;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  const int G = cache->num_kv_heads, d = cache->head_dim;
  const void* k = layer_pool(cache, cache->k_pool, layer);
  const void* v = layer_pool(cache, cache->v_pool, layer);
  AttnMaps maps;
  if (!make_attn_maps_strided(&maps, d_q, T, q_row_stride, q_head_stride, k, v,
                              static_cast<long long>(cache->num_blocks) * G * 16, num_heads, G, d, lc.f16))
    return AXON_ERR_UNSUPPORTED;
  ChunkArgs a;
  memset(&a, 0, sizeof(a));
  a.cu = d_cu_seqlens;
  a.past = d_context_lens;
  a.block_table = d_block_table;
  a.blocks_per_seq = blocks_per_seq;
  a.num_blocks = cache->num_blocks;
  a.B = B;
  a.T = T;
  a.max_chunk = max_chunk;
  a.H = num_heads;
  a.G = G;
  a.d = d;
  a.window = window;
  a.sinks = window > 0 ? clamp_sinks(sinks, blocks_per_seq) : 0;
  a.scale_log2 = scale_log2(scale, d);
  a.o = d_out;
  a.o_row = out_row_stride;
  a.o_head = out_head_stride;
  a.err = d_err;
  return status(with_limits([&] { return launch_attn_chunk(lc, a, maps); }));
}

int axon_rope_table(float* d_rope, int32_t positions, int32_t rotary_dim, float theta, float factor, float low, float high,
                    int32_t original_positions, void* stream) {
  if (!d_rope || unaligned(d_rope) || positions < 1 || rotary_dim < 1) return AXON_ERR_INVALID_ARG;
  if (!(theta > 0.f) || isinf(theta) || !(factor >= 0.f) || isinf(factor)) return AXON_ERR_INVALID_ARG;
  if (factor > 0.f && (original_positions <= 0 || !(low > 0.f) || !(high > low) || isinf(high))) return AXON_ERR_INVALID_ARG;
  if (rotary_dim % 16 || rotary_dim > 128) return AXON_ERR_UNSUPPORTED;
  LaunchCtx lc;
  const int rc = launch_ctx(nullptr, stream, &lc);
  if (rc) return rc;
  double f[64];
  for (int j = 0; j < rotary_dim / 2; ++j) f[j] = rope_frequency(theta, rotary_dim, j, factor, low, high, original_positions);
  return status(launch_rope_table(lc, d_rope, positions, rotary_dim / 2, f));
}

int axon_kv_append(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride, int64_t q_head_stride,
                   const void* d_k, int64_t k_row_stride, int64_t k_head_stride, const void* d_v, int64_t v_row_stride,
                   int64_t v_head_stride, int32_t B, int32_t T, int32_t num_heads, const int32_t* d_cu_seqlens,
                   const int32_t* d_context_lens, const int32_t* d_block_table, int32_t blocks_per_seq, const float* d_rope,
                   int32_t rope_positions, int32_t rotary_dim, int32_t rope_layout, void* d_q_out, int64_t out_row_stride,
                   int64_t out_head_stride, int32_t* d_err, void* stream) {
  int rc = check_cache(cache);
  if (rc) return rc;
  const int G = cache->num_kv_heads, d = cache->head_dim;
  if (layer < 0 || layer >= cache->num_layers || !d_k || !d_v || unaligned(d_k) || unaligned(d_v)) return AXON_ERR_INVALID_ARG;
  if (B < 1 || T < 1 || num_heads < 0 || !d_context_lens || (!d_cu_seqlens && T != B)) return AXON_ERR_INVALID_ARG;
  if (blocks_per_seq < 1 || blocks_per_seq > MAX_BLOCKS_PER_SEQ) return AXON_ERR_INVALID_ARG;
  if (!d_block_table && static_cast<long long>(B) * blocks_per_seq > cache->num_blocks) return AXON_ERR_INVALID_ARG;
  if (rotary_dim < 0 || rotary_dim > d || (rotary_dim > 0) != (d_rope != nullptr) || unaligned(d_rope))
    return AXON_ERR_INVALID_ARG;
  if (rotary_dim > 0 && (rope_positions < 1 || (rope_layout != AXON_ROPE_HALF && rope_layout != AXON_ROPE_INTERLEAVED)))
    return AXON_ERR_INVALID_ARG;
  if ((num_heads > 0) != (d_q != nullptr) || (d_q != nullptr) != (d_q_out != nullptr) || unaligned(d_q) || unaligned(d_q_out))
    return AXON_ERR_INVALID_ARG;
  if ((rc = check_strides(T, G, d, k_row_stride, k_head_stride)) || (rc = check_strides(T, G, d, v_row_stride, v_head_stride)))
    return rc;
  if (d_q && ((rc = check_strides(T, num_heads, d, q_row_stride, q_head_stride)) ||
              (rc = check_strides(T, num_heads, d, out_row_stride, out_head_stride))))
    return rc;
  if (d_q && d_q == d_q_out && (q_row_stride != out_row_stride || q_head_stride != out_head_stride)) return AXON_ERR_INVALID_ARG;
  if (rotary_dim % 16 || num_heads > 65536 || G > 65536) return AXON_ERR_UNSUPPORTED;
  LaunchCtx lc;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  AppendArgs a;
  memset(&a, 0, sizeof(a));
  const void* x[3] = {d_q, d_k, d_v};
  const int64_t rows[3] = {q_row_stride, k_row_stride, v_row_stride}, heads[3] = {q_head_stride, k_head_stride, v_head_stride};
  for (int i = 0; i < 3; ++i) {
    a.x[i] = x[i];
    a.x_row[i] = rows[i];
    a.x_head[i] = heads[i];
  }
  a.o = d_q_out;
  a.o_row = out_row_stride;
  a.o_head = out_head_stride;
  a.k = layer_pool(cache, cache->k_pool, layer);
  a.v = layer_pool(cache, cache->v_pool, layer);
  a.cu = d_cu_seqlens;
  a.past = d_context_lens;
  a.block_table = d_block_table;
  a.blocks_per_seq = blocks_per_seq;
  a.num_blocks = cache->num_blocks;
  a.B = B;
  a.T = T;
  a.H = num_heads;
  a.G = G;
  a.d = d;
  a.most = blocks_per_seq * 16;
  if (rotary_dim > 0 && rope_positions < a.most) a.most = rope_positions;
  a.rope = d_rope;
  a.rotary = rotary_dim;
  a.interleaved = rope_layout == AXON_ROPE_INTERLEAVED;
  a.err = d_err;
  return status(launch_append(lc, a, cache->precision == AXON_FP32_DEBUG ? 4 : 2));
}

int axon_kv_workspace(const axon_kv_cache* cache, const axon_kv_seqs* seqs, int64_t* bytes) {
  PagesArgs a;
  if (!seqs || !bytes) return AXON_ERR_INVALID_ARG;
  const int rc = pages_args(cache, seqs, nullptr, -1, nullptr, &a);
  if (rc) return rc;
  *bytes = 4 * static_cast<int64_t>(pages_work_ints(a.N, a.R, a.P));
  return AXON_OK;
}

int axon_kv_copy_blocks(const axon_kv_cache* cache, const int32_t* d_src, const int32_t* d_dst, int32_t n,
                        int32_t* d_err, void* stream) {
  PagesArgs a;
  LaunchCtx lc;
  int rc = pages_args(cache, nullptr, nullptr, -1, d_err, &a);
  if (rc) return rc;
  if (n < 0 || (n > 0 && (!d_src || !d_dst))) return AXON_ERR_INVALID_ARG;
  if (n == 0) return AXON_OK;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  return status(launch_pages_copy(lc, a, d_src, d_dst, n));
}

int axon_kv_fork(const axon_kv_cache* cache, const axon_kv_seqs* seqs, const int32_t* d_src, const int32_t* d_dst,
                 int32_t n, void* d_workspace, int64_t workspace_bytes, int32_t* d_err, void* stream) {
  PagesArgs a;
  LaunchCtx lc;
  if (!seqs || workspace_bytes < 0) return AXON_ERR_INVALID_ARG;
  int rc = pages_args(cache, seqs, d_workspace, workspace_bytes, d_err, &a);
  if (rc) return rc;
  if (n < 0 || n > a.R || (n > 0 && (!d_src || !d_dst))) return AXON_ERR_INVALID_ARG;
  if (n == 0) return AXON_OK;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  return status(launch_pages_fork(lc, a, d_src, d_dst, n));
}

int axon_kv_release(const axon_kv_cache* cache, const axon_kv_seqs* seqs, const int32_t* d_rows, int32_t n,
                    int32_t window, int32_t sinks, int32_t* d_err, void* stream) {
  PagesArgs a;
  LaunchCtx lc;
  if (!seqs) return AXON_ERR_INVALID_ARG;
  int rc = pages_args(cache, seqs, nullptr, -1, d_err, &a);
  if (rc) return rc;
  if (n < 0 || n > a.R || window < 0 || sinks < 0) return AXON_ERR_INVALID_ARG;
  if (n == 0) return AXON_OK;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  return status(launch_pages_release(lc, a, d_rows, n, window > 0 ? window : -1, clamp_sinks(sinks, a.P)));
}

int axon_kv_reserve(const axon_kv_cache* cache, const axon_kv_seqs* seqs, const int32_t* d_rows,
                    const int32_t* d_new_tokens, int32_t n, void* d_workspace, int64_t workspace_bytes,
                    int32_t* d_err, void* stream) {
  PagesArgs a;
  LaunchCtx lc;
  if (!seqs || workspace_bytes < 0) return AXON_ERR_INVALID_ARG;
  int rc = pages_args(cache, seqs, d_workspace, workspace_bytes, d_err, &a);
  if (rc) return rc;
  if (n < 0 || n > a.R || (n > 0 && !d_new_tokens)) return AXON_ERR_INVALID_ARG;
  if (n == 0) return AXON_OK;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  return status(launch_pages_reserve(lc, a, d_rows, d_new_tokens, n));
}

int axon_kv_compact(const axon_kv_cache* cache, const axon_kv_seqs* seqs, int32_t* d_moved, int32_t* d_live,
                    void* d_workspace, int64_t workspace_bytes, int32_t* d_err, void* stream) {
  PagesArgs a;
  LaunchCtx lc;
  if (!seqs || workspace_bytes < 0) return AXON_ERR_INVALID_ARG;
  int rc = pages_args(cache, seqs, d_workspace, workspace_bytes, d_err, &a);
  if (rc) return rc;
  if ((rc = launch_ctx(cache, stream, &lc))) return rc;
  return status(launch_pages_compact(lc, a, d_moved, d_live));
}

int axon_sample(const void* d_logits, int64_t row_stride, int32_t precision, int32_t B, int32_t V, const float* d_temperature,
                const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, const float* d_u, int32_t* d_tokens,
                float* d_prob, void* stream) {
  if (!d_logits || !d_u || !d_tokens || B < 1 || V < 1 || (B > 1 && row_stride < V)) return AXON_ERR_INVALID_ARG;
  if (precision != AXON_BF16 && precision != AXON_FP16 && precision != AXON_FP32_DEBUG) return AXON_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d_logits) % (precision == AXON_FP32_DEBUG ? 4 : 2)) return AXON_ERR_INVALID_ARG;
  if (V > SAMPLE_MAX_VOCAB || B > SAMPLE_MAX_ROWS) return AXON_ERR_UNSUPPORTED;
  LaunchCtx lc;
  const int rc = launch_ctx(nullptr, stream, &lc);
  if (rc) return rc;
  SampleArgs a;
  memset(&a, 0, sizeof(a));
  a.logits = d_logits;
  a.row_stride = row_stride;
  a.B = B;
  a.V = V;
  a.temperature = d_temperature;
  a.top_k = d_top_k;
  a.top_p = d_top_p;
  a.min_p = d_min_p;
  a.u = d_u;
  a.tokens = d_tokens;
  a.prob = d_prob;
  return status(with_limits([&] { return launch_sample(lc, a, precision); }));
}

int axon_check_error(int32_t* d_err, void* stream, int32_t* bits) {
  if (!d_err) return AXON_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t v = 0;
  cudaError_t e = cudaMemcpyAsync(&v, d_err, sizeof(v), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(d_err, 0, sizeof(v), st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return status(e);
  if (bits) *bits = v;
  if (v & DEVERR_TIMEOUT) return AXON_ERR_TIMEOUT;
  return v ? AXON_ERR_DEVICE_CHECK : AXON_OK;
}

}  // extern "C"
