// C ABI of the coded KV cache (nq_kv_append, nq_attend): argument checks and dispatch.  The
// declarations and their contracts are in include/nestquant.h.
#include <algorithm>
#include <cmath>

#include "nestquant.h"
#include "nq_device_once.hpp"
#include "nq_kernels.hpp"

namespace {

using nq::set_error;

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
int64_t dtype_size(nq_dtype d) { return d == NQ_F32 ? 4 : 2; }
bool is_dtype(nq_dtype d) { return d == NQ_F32 || d == NQ_F16 || d == NQ_BF16; }

nq_status done(hipError_t e, const char* who) {
  if (e != hipSuccess) return set_error(NQ_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
  return set_error(NQ_OK, "%s", "");
}

constexpr int64_t kMaxTokens = (int64_t)1 << 31;
constexpr int64_t kMaxThreads = (int64_t)1 << 32;   // of a launch (a HIP grid counts them in 32 bits)

nq_status check_cache(const nq_kv_cache* c, const char* who) {
  if (!c) return set_error(NQ_ERR_INVALID_ARG, "%s: cache is NULL", who);
  if (c->dim != 64 && c->dim != 128 && c->dim != 256)
    return set_error(NQ_ERR_UNSUPPORTED, "%s: dim=%d must be 64, 128 or 256", who, c->dim);
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1)) != 0)
    return set_error(NQ_ERR_UNSUPPORTED, "%s: page=%d must be 16, 32, 64, 128 or 256", who, c->page);
  if (c->heads < 1 || c->heads > 1024)
    return set_error(NQ_ERR_INVALID_ARG, "%s: heads=%d outside [1, 1024]", who, c->heads);
  if (c->pages < 0 || c->pages > ((int64_t)1 << 40) / c->page)
    return set_error(NQ_ERR_INVALID_ARG, "%s: pages=%lld outside [0, 2^40 / page]", who,
                     (long long)c->pages);
  if (c->reserved != 0) return set_error(NQ_ERR_INVALID_ARG, "%s: reserved is not 0", who);
  for (const nq_params* p : {&c->k, &c->v}) {
    if (nq_status s = nq::check_code(p, c->dim, who)) return s;
    if (p->strategy != NQ_FIRST_BETA)
      return set_error(NQ_ERR_UNSUPPORTED, "%s: a cache is coded with First-beta", who);
  }
  if (c->pages > 0) {
    for (const void* p : {(const void*)c->k_codes, (const void*)c->k_beta, (const void*)c->k_scales,
                          (const void*)c->v_codes, (const void*)c->v_beta, (const void*)c->v_scales})
      if (!p || !aligned16(p))
        return set_error(NQ_ERR_INVALID_ARG, "%s: the pools must be 16-byte aligned, not NULL", who);
  }
  return NQ_OK;
}

nq_status check_rows(const nq_heads* x, nq_dtype dtype, const char* name, const char* who) {
  if (!x || !x->data) return set_error(NQ_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
  const int64_t e = dtype_size(dtype);
  if (!aligned16(x->data) || x->token_stride * e % 16 != 0 || x->head_stride * e % 16 != 0 ||
      x->token_stride < 0 || x->head_stride < 0)
    return set_error(NQ_ERR_INVALID_ARG,
                     "%s: %s and its strides must be 16-byte aligned, the strides not negative", who,
                     name);
  return NQ_OK;
}

int log2_of(int v) {
  int l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

// fp16 bits of a whole number of at most 11 significant bits, 0 < |v| < 65504.
uint32_t f16_bits(int v) {
  const uint32_t sign = v < 0 ? 0x8000u : 0u;
  uint32_t u = (uint32_t)(v < 0 ? -v : v);
  int e = 0;
  while ((u >> e) > 1) ++e;
  const uint32_t frac = e <= 10 ? (u << (10 - e)) : (u >> (e - 10));
  return sign | (uint32_t)(e + 15) << 10 | (frac & 0x3FFu);
}

nq::AttendCode attend_code(const nq_params* p) {
  const nq::EncodeArgs e = nq::code_args(p);
  nq::AttendCode c{e.q, e.m2q, 0u, 0u, 0u, 0u};
  for (int i = 0; i < 4; ++i) {
    const int m = (int)((e.mtab >> (8 * i)) & 0xFFu);
    const uint32_t hm = f16_bits(m), hc = f16_bits(-144 * m);
    c.m_lo |= (hm & 0xFFu) << (8 * i);
    c.m_hi |= (hm >> 8) << (8 * i);
    c.c_lo |= (hc & 0xFFu) << (8 * i);
    c.c_hi |= (hc >> 8) << (8 * i);
  }
  return c;
}

nq_status check_attend(int32_t heads, int32_t dim, int64_t tokens, int32_t q_heads, int64_t seqs,
                       int64_t max_queries, int64_t max_length, int64_t window, int64_t sinks,
                       const char* who) {
  if (heads < 1 || heads > 1024 || (dim != 64 && dim != 128 && dim != 256))
    return set_error(NQ_ERR_INVALID_ARG, "%s: heads or dim out of range", who);
  if (q_heads < 1 || q_heads % heads != 0 || q_heads / heads > 1024)
    return set_error(NQ_ERR_INVALID_ARG,
                     "%s: q_heads=%d must be a multiple of heads=%d, at most 1024 times it", who,
                     q_heads, heads);
  if (tokens < 0 || tokens * q_heads >= kMaxTokens)
    return set_error(NQ_ERR_INVALID_ARG, "%s: tokens * q_heads outside [0, 2^31)", who);
  if (seqs < 0 || seqs > 65535)
    return set_error(NQ_ERR_INVALID_ARG, "%s: seqs=%lld outside [0, 65535]", who, (long long)seqs);
  // a call of no tokens is a no-op whatever its bounds allow
  if (max_queries < 0 || (tokens > 0 && max_queries > tokens))
    return set_error(NQ_ERR_INVALID_ARG, "%s: max_queries outside [0, tokens]", who);
  if (max_length < 0 || max_length >= ((int64_t)1 << 30))
    return set_error(NQ_ERR_INVALID_ARG, "%s: max_length outside [0, 2^30)", who);
  if (window < 0 || sinks < 0)
    return set_error(NQ_ERR_INVALID_ARG, "%s: window and sinks must not be negative", who);
  return NQ_OK;
}

// Tiles of `size` tokens that n consecutive queries may see.  It grows with every argument (window
// 0 counting as the largest) but size.
int64_t seen_tiles(int64_t size, int64_t n, int64_t max_length, int64_t window, int64_t sinks) {
  const int64_t whole = (max_length + size - 1) / size;
  if (window == 0) return whole;
  const int64_t w = std::min(window, max_length), s = std::min(sinks, max_length);
  return std::min(whole, (w + n) / size + 2 + (s + size - 1) / size);
}

// Bytes of a partial row (the maximum, the sum, two unused floats, dim entries) and of a record.
int64_t part_bytes(int dim) { return (int64_t)(dim + 4) * 4; }
int64_t record_bytes(int dim) { return (int64_t)dim * 256 + 1024; }

}  // namespace

nq::AttendPlan nq::attend_plan(int heads, int dim, int64_t tokens, int q_heads, int64_t seqs,
                               int64_t max_queries, int64_t max_length, int64_t window,
                               int64_t sinks) {
  (void)tokens;
  const int64_t group = q_heads / heads, rows = max_queries * group;
  AttendPlan p{};
  p.tiles = rows > 64 ? 0 : (rows > 16 && dim < 256 ? 2 : 1);
  const int64_t most = p.tiles == 0 ? 128 : 16 * p.tiles;
  p.blocks = (int)((rows + most - 1) / most);
  p.rows = (int)std::min(rows, most);
  auto tiles = [&](int64_t size, int64_t n) { return seen_tiles(size, n, max_length, window, sinks); };
  const int64_t queries = std::min(max_queries, most / group + 2);   // of a row block
  const int64_t wgs = std::max<int64_t>(seqs * heads * p.blocks, 1);
  if (p.tiles == 0) {
    p.groups = (int)std::max<int64_t>(tiles(64, max_queries), 1);
    const int64_t steps = std::max<int64_t>(tiles(64, queries), 1);
    const int64_t chunks = std::max<int64_t>(std::min((512 + wgs - 1) / wgs, (steps + 7) / 8), 1);
    p.steps = (int)((steps + chunks - 1) / chunks);
    p.chunks = (int)((steps + p.steps - 1) / p.steps);
  } else {
    // One tile of 16 tokens a step while that leaves every tile a wave of its own on the chip's
    // 1024 SIMDs, which halves what a wave does: 391 tokens of 8 KV heads 11.4 -> 9.9 us, 1000
    // tokens of 256 entries 17.2 -> 13.3; past it 4000 tokens took 17.9 -> 21.7 us (256 entries),
    // 4 x 1000 tokens 12.7 -> 13.6.  Up to eight tiles are one chunk, with no join, either way.
    const int64_t all = std::max<int64_t>(tiles(16, queries), 1);
    p.units = p.tiles == 1 && all > 8 && wgs * all <= 1024 ? 1 : 2;
    const int64_t steps = (all + p.units - 1) / p.units;
    int64_t chunks = std::max((2048 + wgs - 1) / wgs, (steps + 15) / 16);
    chunks = std::max<int64_t>(std::min(chunks, (steps + 3) / 4), 1);
    p.steps = (int)((steps + chunks - 1) / chunks);
    p.steps = (p.steps + 3) / 4 * 4;
    p.chunks = (int)((steps + p.steps - 1) / p.steps);
  }
  const int64_t records = seqs * heads * p.groups;       // one a workgroup
  const int64_t parts = wgs * p.rows;                    // rows that are joined, some a workgroup
  const int64_t joins = p.chunks > 1 ? parts / (1024 / dim) + 1 : 0;
  p.fits = std::max({wgs * p.chunks, records, joins}) * 256 < kMaxThreads && parts < kMaxTokens;
  if (!p.fits) return p;
  p.records = records * record_bytes(dim);
  p.part = p.chunks > 1 ? parts * p.chunks * part_bytes(dim) : 0;
  return p;
}

extern "C" {

nq_status nq_kv_append(const nq_kv_cache* cache, const nq_kv_prep* prep, int64_t tokens,
                       const int64_t* slots, const int32_t* positions, nq_dtype dtype,
                       const nq_heads* q, int32_t q_heads, const nq_heads* k, const nq_heads* v,
                       const nq_heads* q_out, nq_dtype out_dtype, void* hip_stream) {
  const char* who = "nq_kv_append";
  if (nq_status s = check_cache(cache, who)) return s;
  if (!prep) return set_error(NQ_ERR_INVALID_ARG, "%s: prep is NULL", who);
  if (!is_dtype(dtype) || (q_heads > 0 && !is_dtype(out_dtype)))
    return set_error(NQ_ERR_UNSUPPORTED, "%s: unsupported dtype", who);
  if (prep->rot < 0 || prep->rot > cache->dim || prep->rot % 16 != 0)
    return set_error(NQ_ERR_INVALID_ARG, "%s: rot=%d must be a multiple of 16 in [0, dim]", who,
                     prep->rot);
  if (prep->pairs != NQ_PAIRS_HALVES && prep->pairs != NQ_PAIRS_NEIGHBOURS)
    return set_error(NQ_ERR_INVALID_ARG, "%s: pairs=%d is not an nq_pairs", who, prep->pairs);
  if (prep->hadamard != 0 && prep->hadamard != 1)
    return set_error(NQ_ERR_INVALID_ARG, "%s: hadamard must be 0 or 1", who);
  if (prep->reserved != 0) return set_error(NQ_ERR_INVALID_ARG, "%s: reserved is not 0", who);
  if ((prep->q_norm || prep->k_norm) && !(prep->eps >= 0.0 && std::isfinite(prep->eps)))
    return set_error(NQ_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", who);
  if (prep->rot > 0) {
    if (!prep->cos || !prep->sin || !aligned16(prep->cos) || !aligned16(prep->sin))
      return set_error(NQ_ERR_INVALID_ARG, "%s: cos and sin must be 16-byte aligned, not NULL", who);
    if (prep->positions < 1 || prep->positions >= kMaxTokens)
      return set_error(NQ_ERR_INVALID_ARG, "%s: the tables' positions outside [1, 2^31)", who);
  }
  if (q_heads < 0 || tokens < 0 || tokens >= kMaxTokens || tokens * cache->heads >= kMaxTokens ||
      tokens * q_heads >= kMaxTokens)
    return set_error(NQ_ERR_INVALID_ARG, "%s: tokens times heads outside [0, 2^31)", who);
  // 256 blocks a workgroup of 64 threads, queries beside keys and values up to 2^23 blocks
  const int64_t nb = cache->dim / 8, q_blocks = tokens * q_heads * nb;
  const int64_t wgs = 2 * ((tokens * cache->heads * nb + 255) / 256) +
                      (q_blocks < (int64_t)1 << 23 ? (q_blocks + 255) / 256 : 0);
  if (wgs * 64 >= kMaxThreads)
    return set_error(NQ_ERR_UNSUPPORTED, "%s: more workgroups than a launch holds", who);
  if (tokens == 0) return done(hipSuccess, who);
  if (!slots || (prep->rot > 0 && !positions))
    return set_error(NQ_ERR_INVALID_ARG, "%s: slots or positions is NULL", who);
  if (nq_status s = check_rows(k, dtype, "k", who)) return s;
  if (nq_status s = check_rows(v, dtype, "v", who)) return s;
  if (q_heads > 0) {
    if (nq_status s = check_rows(q, dtype, "q", who)) return s;
    if (nq_status s = check_rows(q_out, out_dtype, "q_out", who)) return s;
  }
  nq::KVAppendArgs a{};
  a.k = {k->data, k->token_stride, k->head_stride};
  a.v = {v->data, v->token_stride, v->head_stride};
  if (q_heads > 0) {
    a.q = {q->data, q->token_stride, q->head_stride};
    a.out = {q_out->data, q_out->token_stride, q_out->head_stride};
  }
  a.pk = {cache->k_codes, cache->k_beta, cache->k_scales};
  a.pv = {cache->v_codes, cache->v_beta, cache->v_scales};
  a.ck = nq::code_args(&cache->k);
  a.cv = nq::code_args(&cache->v);
  a.slots = slots;
  a.positions = positions;
  a.cos = prep->cos;
  a.sin = prep->sin;
  a.q_norm = prep->q_norm;
  a.k_norm = prep->k_norm;
  a.eps = prep->eps;
  a.limit = cache->pages * cache->page;
  a.tokens = (int)tokens;
  a.q_heads = q_heads;
  a.heads = cache->heads;
  a.table_rows = (int)prep->positions;
  a.rot = prep->rot;
  a.pairs = prep->pairs;
  a.hadamard = prep->hadamard;
  a.page_shift = log2_of(cache->page);
  a.out_dtype = (int)out_dtype;
  a.rot_s = (float)(1.0 / std::sqrt((double)cache->dim));   // as nq_rotate's scaling
  a.by_q = nq::row_divisor(q_heads > 0 ? (uint32_t)q_heads : 1u);
  a.by_kv = nq::row_divisor((uint32_t)cache->heads);
  return done(nq::launch_kv_append(a, (int)dtype, cache->dim, (hipStream_t)hip_stream), who);
}

int64_t nq_attend_workspace_size(int32_t heads, int32_t dim, int64_t tokens, int32_t q_heads,
                                 int64_t seqs, int64_t max_queries, int64_t max_length,
                                 int64_t window, int64_t sinks) {
  if (check_attend(heads, dim, tokens, q_heads, seqs, max_queries, max_length, window, sinks,
                   "nq_attend_workspace_size"))
    return -1;
  if (tokens == 0 || seqs == 0 || max_queries == 0) return 0;
  const nq::AttendPlan p = nq::attend_plan(heads, dim, tokens, q_heads, seqs, max_queries,
                                           max_length, window, sinks);
  return p.fits ? p.part + p.records : -1;
}

// What no plan of smaller arguments exceeds.  The sizes themselves are not monotone: fewer rows or
// sequences are split into more chunks, and a chunk's steps are rounded.
int64_t nq_attend_workspace_bound(int32_t heads, int32_t dim, int64_t tokens, int32_t q_heads,
                                  int64_t seqs, int64_t max_queries, int64_t max_length,
                                  int64_t window, int64_t sinks) {
  if (check_attend(heads, dim, tokens, q_heads, seqs, max_queries, max_length, window, sinks,
                   "nq_attend_workspace_bound"))
    return -1;
  if (tokens == 0 || seqs == 0 || max_queries == 0) return 0;
  if (!nq::attend_plan(heads, dim, tokens, q_heads, seqs, max_queries, max_length, window, sinks).fits)
    return -1;
  const int64_t group = q_heads / heads, rows = max_queries * group, pairs = seqs * heads;
  int64_t few = 0, many = 0;
  {
    // Few rows: at most 64 a pair, in blocks of 16 or 32 (padded to 32 from 17 on); chunks n with
    //   blocks pairs n <= max(2048 + blocks pairs, blocks pairs ceil(steps / 16)),
    // n <= ceil(tiles / 4), and one where there are no more than eight tiles.
    const int64_t r = std::min<int64_t>(rows, 64), block = dim < 256 ? 32 : 16;
    const int64_t padded = r <= 16 ? r : (r + 31) / 32 * 32, blocks = (r + 15) / 16;
    const int64_t all = seen_tiles(16, std::min(max_queries, 32 / group + 2), max_length, window, sinks);
    const int64_t wgs = pairs * blocks, chunks = (all + 3) / 4;
    if (all > 8)
      few = std::min(std::max(2048 + wgs, wgs * (((all + 1) / 2 + 15) / 16)) * std::min(r, block),
                     pairs * padded * chunks);
  }
  if (rows > 64) {
    // Many: blocks of 128 rows; more than one chunk below 512 blocks and above 8 records only.
    const int64_t wgs = std::min<int64_t>(pairs * ((rows + 127) / 128), 511);
    const int64_t steps = seen_tiles(64, std::min(max_queries, 128 / group + 2), max_length, window, sinks);
    if (steps > 8) many = std::min(511 + wgs, wgs * ((steps + 7) / 8)) * std::min<int64_t>(rows, 128);
  }
  const int64_t records =
      rows > 64 ? pairs * std::max<int64_t>(seen_tiles(64, max_queries, max_length, window, sinks), 1) : 0;
  return std::max(few * part_bytes(dim), many * part_bytes(dim) + records * record_bytes(dim));
}

nq_status nq_attend(const nq_kv_cache* cache, const int32_t* table, int64_t table_stride,
                    const int32_t* lengths, int64_t seqs, const int32_t* starts,
                    int64_t max_queries, int64_t max_length, int64_t window, int64_t sinks,
                    double scale, nq_dtype dtype, const nq_heads* q, int64_t tokens,
                    int32_t q_heads, const nq_heads* out, float* lse, void* workspace,
                    int64_t workspace_bytes, void* hip_stream) {
  const char* who = "nq_attend";
  if (nq_status s = check_cache(cache, who)) return s;
  if (cache->k.decoder != cache->v.decoder)
    return set_error(NQ_ERR_UNSUPPORTED, "%s: keys and values with different decoders", who);
  if (!is_dtype(dtype)) return set_error(NQ_ERR_UNSUPPORTED, "%s: unsupported dtype", who);
  if (nq_status s = check_attend(cache->heads, cache->dim, tokens, q_heads, seqs, max_queries,
                                 max_length, window, sinks, who))
    return s;
  const float k_scale = (float)(scale * 1.4426950408889634 * cache->k.base * 4.0);
  if (!std::isfinite(scale) || !std::isfinite(k_scale))
    return set_error(NQ_ERR_INVALID_ARG, "%s: scale is not finite in fp32", who);
  if (table_stride < 0 || max_length > table_stride * cache->page)
    return set_error(NQ_ERR_INVALID_ARG, "%s: max_length exceeds table_stride * page", who);
  if (cache->pages >= kMaxTokens)
    return set_error(NQ_ERR_INVALID_ARG, "%s: a page table names fewer than 2^31 pages", who);
  if (!starts && tokens != seqs)
    return set_error(NQ_ERR_INVALID_ARG, "%s: without starts there is one query a sequence", who);
  if (tokens == 0 || seqs == 0 || max_queries == 0) return done(hipSuccess, who);
  if (!lengths || (max_length > 0 && !table))
    return set_error(NQ_ERR_INVALID_ARG, "%s: table or lengths is NULL", who);
  if (nq_status s = check_rows(q, dtype, "q", who)) return s;
  if (nq_status s = check_rows(out, dtype, "out", who)) return s;
  const nq::AttendPlan p = nq::attend_plan(cache->heads, cache->dim, tokens, q_heads, seqs,
                                           max_queries, max_length, window, sinks);
  if (!p.fits)
    return set_error(NQ_ERR_UNSUPPORTED, "%s: more workgroups than a launch holds", who);
  const int64_t need = p.part + p.records;
  if (workspace_bytes < need || (need > 0 && (!workspace || !aligned16(workspace))))
    return set_error(NQ_ERR_INVALID_ARG, "%s: workspace of %lld bytes needed, 16-byte aligned", who,
                     (long long)need);
  nq::AttendArgs a{};
  a.k = {cache->k_codes, cache->k_beta, cache->k_scales};
  a.v = {cache->v_codes, cache->v_beta, cache->v_scales};
  a.ck = attend_code(&cache->k);
  a.cv = attend_code(&cache->v);
  a.table = table;
  a.lengths = lengths;
  a.starts = starts;
  a.table_stride = table_stride;
  a.pages = cache->pages;
  a.q = {q->data, q->token_stride, q->head_stride};
  a.out = out->data;
  a.out_token = out->token_stride;
  a.out_head = out->head_stride;
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  a.records = static_cast<unsigned char*>(workspace) + p.part;
  a.groups = p.groups;
  const int64_t wgs = (int64_t)p.chunks * p.blocks * cache->heads * seqs;
  a.mirror = p.chunks == 1 && p.blocks % 2 == 0 && wgs <= 512;
  a.k_scale = k_scale;
  a.v_scale = (float)(cache->v.base * 4.0);
  a.seqs = (int)seqs;
  a.tokens = (int)tokens;
  a.max_queries = (int)max_queries;
  // an empty pool holds nothing to see (and nothing to read)
  a.max_length = cache->pages > 0 ? (int)max_length : 0;
  a.window = (int)std::min<int64_t>(window, (int64_t)1 << 30);
  a.sinks = (int)std::min<int64_t>(sinks, (int64_t)1 << 30);
  a.heads = cache->heads;
  a.q_heads = q_heads;
  a.page_shift = log2_of(cache->page);
  a.dtype = (int)dtype;
  a.blocks = p.blocks;
  a.rows = p.rows;
  a.chunks = p.chunks;
  a.steps = p.steps;
  a.by_group = nq::row_divisor((uint32_t)(q_heads / cache->heads));
  a.by_q = nq::row_divisor((uint32_t)q_heads);
  hipStream_t st = (hipStream_t)hip_stream;
  static nq::PerDevice few(nq::attend_set_attributes), many(nq::prompt_set_attributes);
  const hipError_t e = (p.tiles ? few : many).ensure(st);
  if (e != hipSuccess) return done(e, who);
  return done(p.tiles ? nq::launch_attend(a, p, cache->dim, cache->k.decoder, st)
                      : nq::launch_prompt(a, cache->dim, cache->k.decoder, st),
              who);
}

}  // extern "C"
