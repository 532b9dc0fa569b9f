// What the attention kernels over a coded KV cache share: the call's arguments, which tiles of
// the cache a block of queries sees, and the decode of code words into fp16 matrix operands.
#pragma once

#include "nq_device.hpp"
#include "nq_kernels.hpp"

namespace nq {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// A sequence's queries and the tokens of the cache they may see.
struct Sequence {
  int first;     // its first row of q
  int queries;   // rows that are computed
  int shift;     // position of query i: shift + i
  int end;       // tokens past the last one that is read
};

__device__ __forceinline__ Sequence sequence_of(const AttendArgs& a, int b) {
  Sequence s;
  int lo = b, hi = b + 1;
  if (a.starts) {
    lo = a.starts[b];
    hi = a.starts[b + 1];
    lo = lo < 0 ? 0 : (lo > a.tokens ? a.tokens : lo);
    hi = hi < lo ? lo : (hi > a.tokens ? a.tokens : hi);
  }
  int n = a.lengths[b];
  n = n < 0 ? 0 : (n > (1 << 30) ? (1 << 30) : n);
  s.first = lo;
  s.queries = hi - lo < a.max_queries ? hi - lo : a.max_queries;
  s.shift = n - (hi - lo);
  s.end = n < a.max_length ? n : a.max_length;
  return s;
}

// Tiles of 2^SHIFT tokens that queries at positions p_lo .. p_hi see, in order: `sink` tiles from
// token 0 on, then those from tile `first` on, `count` in all.
struct Tiles {
  int sink, first, count;
  __device__ int tile(int u) const { return u < sink ? u : u - sink + first; }
  __device__ int index(int tile) const { return tile < sink ? tile : tile - first + sink; }
};

template <int SHIFT>
__device__ __forceinline__ Tiles tiles_of(const AttendArgs& a, int p_lo, int p_hi, int end) {
  Tiles t;
  if (p_hi >= end) p_hi = end - 1;
  if (p_hi < 0) return {0, 0, 0};
  const int stop = (p_hi >> SHIFT) + 1;
  int low = 0;
  if (a.window > 0 && p_lo >= a.window) low = p_lo - a.window + 1;
  t.first = low >> SHIFT;
  if (t.first > stop) t.first = stop;          // only where the queries outrun the tokens
  const int sinks = a.sinks < end ? a.sinks : end;
  t.sink = (sinks + (1 << SHIFT) - 1) >> SHIFT;
  if (t.sink >= t.first) {
    t.sink = 0;
    t.first = 0;
  }
  t.count = t.sink + stop - t.first;
  return t;
}

// What workgroup `id` of a call's grid works on.  The KV head runs fastest, so that with 8 heads
// (or a multiple) each of the chip's 8 dies keeps one head's tokens in its cache, then the
// sequence, then the part (row block and chunk): sequences end in different parts, and with the
// part fastest the dies that are dealt the late ones ran idle (64 ragged sequences: 475 us,
// 271 for as many tokens in equal ones).
struct Place {
  int head, b, part;
};
__device__ __forceinline__ Place place_of(const AttendArgs& a, uint32_t id) {
  const uint32_t x = id / (uint32_t)a.heads;
  return {(int)(id - x * (uint32_t)a.heads), (int)(x % (uint32_t)a.seqs), (int)(x / (uint32_t)a.seqs)};
}

// A block of BR query rows of one KV head: the sequence's rows r0 .. r0 + rows - 1, those of query
// i and head hq of the group at r = i * group + hq.
struct RowBlock {
  int r0, rows;        // rows that exist, at most BR
  int p_lo, p_hi;      // positions of its first and last query
};
__device__ __forceinline__ int query_of(const AttendArgs& a, int r) {
  return (int)(((uint64_t)(uint32_t)r * a.by_group.magic) >> a.by_group.shift);
}
template <int BR>
__device__ __forceinline__ RowBlock row_block(const AttendArgs& a, const Sequence& s, int rb) {
  RowBlock k;
  k.r0 = rb * BR;
  const int left = s.queries * (int)a.by_group.n - k.r0;
  k.rows = left < BR ? left : BR;
  k.p_lo = s.shift + query_of(a, k.r0);
  k.p_hi = s.shift + query_of(a, k.r0 + (k.rows > 0 ? k.rows - 1 : 0));
  return k;
}
// Partial result of a chunk for row r of a block: its maximum and sum, two unused floats, the
// weighted sum of the values.
__device__ __forceinline__ float* partial(const AttendArgs& a, int b, int head, int rb, int r,
                                          int chunk, int dim) {
  return a.part + (((((int64_t)b * a.heads + head) * a.blocks + rb) * a.rows + r) * a.chunks + chunk) *
                      (dim + 4);
}

// N blocks of eight entries of a query row, STRIDE entries apart, as floats (all loads first).
// WIDE: fp32 queries, else fp16 or bf16.
template <bool WIDE, int N, int STRIDE>
__device__ __forceinline__ void load_query(const void* p, int dtype, int64_t at, float (&x)[N][8]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int s = 0; s < N; ++s) {
      const f32x4* q = reinterpret_cast<const f32x4*>((const float*)p + at + STRIDE * s);
      const f32x4 a = q[0], b = q[1];
#pragma unroll
      for (int l = 0; l < 4; ++l) {
        x[s][l] = a[l];
        x[s][4 + l] = b[l];
      }
    }
  } else {
    u32x4 w[N];
#pragma unroll
    for (int s = 0; s < N; ++s)
      w[s] = *reinterpret_cast<const u32x4*>((const uint16_t*)p + at + STRIDE * s);
    if (dtype == NQ_F16) {
#pragma unroll
      for (int s = 0; s < N; ++s) {
        const h8 v = __builtin_bit_cast(h8, w[s]);
#pragma unroll
        for (int l = 0; l < 8; ++l) x[s][l] = (float)v[l];
      }
    } else {
#pragma unroll
      for (int s = 0; s < N; ++s)
#pragma unroll
        for (int l = 0; l < 4; ++l) {
          x[s][2 * l] = __uint_as_float(w[s][l] << 16);
          x[s][2 * l + 1] = __uint_as_float(w[s][l] & 0xFFFF0000u);
        }
    }
  }
}

// The tokens a query sees: `count` from token `low` on, and those before `sinks`.
struct Range {
  int low, count, sinks;
  __device__ bool sees(int j) const { return ((uint32_t)(j - low) < (uint32_t)count) | (j < sinks); }
};
__device__ __forceinline__ Range range_of(const AttendArgs& a, int pos, int end) {
  Range r;
  const int last = pos < end ? pos : end - 1;
  r.low = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  r.count = last >= r.low ? last - r.low + 1 : 0;
  r.sinks = a.sinks <= last ? a.sinks : last + 1;
  return r;
}

__device__ __forceinline__ void store_out(void* p, int dtype, int64_t i, f32x4 v) {
  if (dtype == NQ_F32) {
    *reinterpret_cast<f32x4*>((float*)p + i) = v;
  } else if (dtype == NQ_F16) {
    *reinterpret_cast<h4*>((_Float16*)p + i) = __builtin_convertvector(v, h4);
  } else {
    typedef __bf16 b4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<b4*>((__bf16*)p + i) = __builtin_convertvector(v, b4);
  }
}

// The code words and beta indices of a lane's blocks: NBL blocks from block NBL * g of row
// `row` on, and the row's beta word from their index on.
template <int NBL>
struct Words {
  uint32_t w[NBL];
  uint32_t beta;
};
template <int NBL>
__device__ __forceinline__ Words<NBL> load_words(const AttendPool& p, int64_t row, int g) {
  Words<NBL> r;
  const uint32_t* __restrict__ c = p.codes + row * (4 * NBL) + NBL * g;
  if constexpr (NBL == 2) {
    const u32x2 a = *reinterpret_cast<const u32x2*>(c);
    r.w[0] = a.x; r.w[1] = a.y;
  } else {
#pragma unroll
    for (int i = 0; i < NBL; i += 4) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(c + i);
      r.w[i] = a.x; r.w[i + 1] = a.y; r.w[i + 2] = a.z; r.w[i + 3] = a.w;
    }
  }
  if constexpr (NBL == 8) {
    r.beta = p.beta[row * 2 + (g >> 1)] >> (16 * (g & 1));
  } else {
    r.beta = p.beta[row] >> (2 * NBL * g);
  }
  return r;
}

// Four tokens of one column of a row-major fp16 tile in LDS: the 16 lanes of a group name rows
// 4 x 16 entries (lane i row i / 4, entries 4 (i % 4) ..) and get column i of them.
__device__ __forceinline__ h4 read_transposed(const _Float16* p) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s4 lds_s4;
  return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                    (lds_s4*)(__attribute__((address_space(3))) void*)p));
}

// w as the fp32 number it is: without this the compiler may round a product to fp16 in one step in
// one place and in two in another, and the first of two fp16 terms is then not the one that
// the second completes (single weights were off by 2^-11).
__device__ __forceinline__ float settled(float w) {
  asm("" : "+v"(w));
  return w;
}

// The pair (a, b) as the sum of two fp16 pairs (22 bits): the second is what the first leaves, one
// mixed fused multiply-add an entry (exact) from the packed pair itself.
__device__ __forceinline__ void two_terms(float a, float b, uint32_t& first, uint32_t& second) {
  first = __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
  float c, d;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(c) : "v"(first), "v"(a));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(first), "v"(b));
  second = __builtin_bit_cast(uint32_t, h2{(_Float16)c, (_Float16)d});
}

// The exponent e of a row's largest entry (clamped so that 2^(14 - e) is a number): its entries
// times 2^(14 - e) are fp16 operands.
__device__ __forceinline__ int row_exponent(float largest) {
  const int e = (int)((__float_as_uint(largest) >> 23) & 0xFFu) - 127;
  return e < -100 ? -100 : e;
}

// |x|, or 0 where that is not a finite number.
__device__ __forceinline__ float finite_size(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;
}

// What a lane keeps of a query row beside its weighted sum of values, o.  With a token's score s
// (base 2) and its value's scale r, l sums 2^(s - m) and o sums 2^(s - ref) r V:
//   m    the largest score so far, short of it by kLag at most;
//   ref  2^(ref + kTop) is the largest product 2^s r so far of the tokens that the row sees, short of
//        it by kRoom at most, so that the products' fp16 operands lie at the top of their type.
// A scale that the row does not see, or whose token has next to no weight, has no part in either.
// Both start below every score.
struct RowSum {
  static constexpr float kTop = 12.0f, kRoom = 3.9f, kLag = 8.0f;
  float m = -3.402823466e38f, l = 0.0f, ref = -3.402823466e38f;
  bool wide = false;   // whether shift() is not 0 in a lane of the wave

  // Whether scores up to s, or products up to 2^(s + lv), may pass what the references allow.
  __device__ __forceinline__ bool passed(float s, float lv) const {
    return (s + lv > ref + (kTop + kRoom)) | (s > m + kLag);
  }
  // Raises the references that the largest score and the largest product (its logarithm) of new
  // tokens pass, which depends on this row alone; the factor of o.  ref stays within 140 below m,
  // which holds every scale that is a normal number.
  __device__ __forceinline__ float raise(float s, float product) {
    const float top = s > m + kLag ? s : m;
    l *= __builtin_amdgcn_exp2f(m - top);
    m = top;
    const float next = fmaxf(product > ref + (kTop + kRoom) ? product - kTop : ref, m - 140.0f);
    const float f = __builtin_amdgcn_exp2f(ref - next);
    ref = next;
    wide = __any(shift() != 0);
    return f;
  }
  // Where the references lie so far apart that 2^(s - ref) may leave fp32's range or lose what l
  // needs, a power of two that brings its products with the scales into it.
  __device__ __forceinline__ int shift() const {
    return ref - m > 30.0f ? 64 : (ref - m < -90.0f ? -64 : 0);
  }
  // What a token with d = s - ref and e = s - m counts in `add`, and its weight w, for any shift.
  __device__ __forceinline__ float term(float d, float e, float r, float& w) const {
    const int h = shift();
    const float p = __builtin_amdgcn_exp2f(d + (float)h);
    w = __builtin_ldexpf(p * r, -h);
    return h ? __builtin_amdgcn_exp2f(e) : p;
  }
  // Adds a sum of 2^(s - ref) (2^(s - m) where there is a shift).
  __device__ __forceinline__ void add(float sum) {
    l = __builtin_fmaf(sum, wide && shift() ? 1.0f : __builtin_amdgcn_exp2f(ref - m), l);
  }
};
// 2^(x / 2); twice as a factor it is 2^x, also where that alone is no normal number.
__device__ __forceinline__ float half_power(float x) { return __builtin_amdgcn_exp2f(0.5f * x); }
// A row that sees nothing has the sum 0 (one whose scores are all not numbers has not).
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? -INFINITY : 0.69314718f * (m + __builtin_amdgcn_logf(l));
}

// Row, in the pools, of a token of one head (the 16 tokens from a multiple of 16 on lie in one
// page, side by side); ok: whether its page is one of the cache's (else a row of page 0).
__device__ __forceinline__ int64_t tile_row(const AttendArgs& a, int b, int head, int token,
                                            bool& ok) {
  const int page = a.table[b * a.table_stride + (token >> a.page_shift)];
  ok = page >= 0 && page < a.pages;
  return ((ok ? (int64_t)page * a.heads + head : head) << a.page_shift) +
         (token & ((1 << a.page_shift) - 1));
}

// The decoded block as eight fp16 values m X2 / 8, exact (|m X2| <= 2048): the biased bytes
// X2 + 128 become the fp16 numbers 128 + byte / 8 by one byte permute for two of them, and one
// packed fma takes m times that minus 144 m.
__device__ __forceinline__ h8 f16_of_bytes(uint32_t xa, uint32_t xb, uint32_t m2, uint32_t c2) {
  auto two = [&](uint32_t x, uint32_t sel) {
    const uint32_t w = __builtin_amdgcn_perm(0x58585858u, x, sel);
    return __builtin_elementwise_fma(__builtin_bit_cast(h2, w), __builtin_bit_cast(h2, m2),
                                     __builtin_bit_cast(h2, c2));
  };
  const h2 a = two(xa, 0x04010400u), b = two(xa, 0x04030402u);
  const h2 c = two(xb, 0x04010400u), d = two(xb, 0x04030402u);
  return h8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

template <bool M>
__device__ __forceinline__ h8 decode_f16(uint32_t word, uint32_t index, const AttendCode& c) {
  // the fp16 pairs (m, m) and (-144 m, -144 m) of the index from tables of their bytes
  const uint32_t sel = __builtin_amdgcn_perm(0u, index, 0x00000000u) | 0x04000400u;
  const uint32_t m2 = __builtin_amdgcn_perm(c.m_hi, c.m_lo, sel);
  const uint32_t c2 = __builtin_amdgcn_perm(c.c_hi, c.c_lo, sel);
  uint32_t xa, xb;
  decode_word_b8<M>(word, c.q, c.m2q, xa, xb);
  return f16_of_bytes(xa, xb, m2, c2);
}

}  // namespace nq
