// Appending to a coded KV cache (nq_kv_append): the rows of new queries, keys and values from
// the projections to where attention reads them, in one launch (queries of many million blocks have
// one of their own).
//
// A lane holds one 8-entry block and a row of NB = dim / 8 blocks takes NB lanes of a wave, so
// every step stays in registers: the norm's sum of squares goes across the lanes of a row by
// DPP, the position rotation takes the other half of its pairs from the same lane or by one
// shuffle, and the Hadamard transform runs its stages h = 1, 2, 4 inside the lane and the
// others across lanes.  Keys and values are then coded as the row encoder does (eval_bytes,
// eval_exact of nq_encode_block.hpp) and written straight to their page.
//
// What bounds it: at one token the chain of dependent steps of a wave (7 us), at thousands the
// encoder's vector instructions for keys and values (720 a wave of 64 blocks with norm and
// rotations, 0.97 a clock of a busy CU: 91-104 us for 16384 tokens of 8 heads); the queries are at
// the limits of both memory and vector issue (64 heads of them: 115-128 us, 4.2-4.7 TB/s, 1.01
// vector instructions a clock of a busy CU).
#include <type_traits>

#include "nq_encode_block.hpp"
#include "nq_kernels.hpp"

namespace nq {
namespace {

// Block held by lane l of a row.  DPP reaches the lanes at distances xor 1, xor 2, xor 7 (the
// mirrored half row) and xor 15 (the mirrored row); with this order of the blocks they hold the
// blocks at xor 1, 2, 4 and 8, the partners of the Hadamard stages h = 8, 16, 32 and 64, so
// that each stage is one DPP operand.
__device__ __forceinline__ int block_of_lane(int l) {
  return (l & 19) ^ ((l & 4) ? 7 : 0) ^ ((l & 8) ? 12 : 0);
}
__device__ __forceinline__ int lane_of_block(int j) {
  return (j & 19) ^ ((j & 4) ? 7 : 0) ^ ((j & 8) ? 15 : 0);
}

template <int H>   // the value of the lane holding the block at xor H / 8
__device__ __forceinline__ float across(float v) {
  if constexpr (H == 128) {
    return __shfl_xor(v, 16, 64);
  } else {
    return __uint_as_float(dpp_across<H / 8>(__float_as_uint(v)));
  }
}

// nq_rotate's transform of a row of 8 NB entries.  Across lanes, the pair (x, p) becomes
// (x + p, p - x); the lane of the second one forms x - p and keeps the sign for the end (both
// partners of a later stage carry it alike, and rounding does not depend on it): one fused
// multiply with +-1, exact before its rounding, a stage.
template <int NB>
__device__ __forceinline__ void hadamard(float (&v)[8], int j, float s) {
#pragma unroll
  for (int h = 1; h < 8; h <<= 1) {
#pragma unroll
    for (int l = 0; l < 8; ++l) {
      if (l & h) continue;
      const float a = v[l], b = v[l + h];
      v[l] = a + b;
      v[l + h] = a - b;
    }
  }
  float sign = 1.0f;
  auto stage = [&](auto h) {
    constexpr int H = decltype(h)::value;
    const float f = (j & (H / 8)) ? -1.0f : 1.0f;
#pragma unroll
    for (int l = 0; l < 8; ++l) v[l] = __builtin_fmaf(across<H>(v[l]), f, v[l]);
    sign *= f;
  };
  stage(std::integral_constant<int, 8>{});
  stage(std::integral_constant<int, 16>{});
  stage(std::integral_constant<int, 32>{});
  if constexpr (NB > 8) stage(std::integral_constant<int, 64>{});
  if constexpr (NB > 16) stage(std::integral_constant<int, 128>{});
  const float f = s * sign;
#pragma unroll
  for (int l = 0; l < 8; ++l) v[l] *= f;
}

__device__ __forceinline__ void load8(const float* __restrict__ p, float (&v)[8]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// The steps of nq_kv_prep on block j of the rows that a lane takes one after another.  What
// they share stays in registers: the norm's weights always, the tables' entries while the
// token is the same (consecutive rows are heads of one token).
template <int NB>
struct RowSteps {
  float w[8];         // the norm's weights
  float c[8], n[8];   // cosines and sines of this lane's pairs, the sines with their sign
  int token;          // whose

  __device__ __forceinline__ void start(const KVAppendArgs& a, const float* __restrict__ weight, int j) {
    token = -1;
    if (weight) load_weights(weight, j);
  }
  __device__ __forceinline__ void load_weights(const float* __restrict__ weight, int j) {
#pragma unroll
    for (int l = 0; l < 8; ++l) w[l] = weight[8 * j + l];
  }
  __device__ __forceinline__ void apply(float (&v)[8], const KVAppendArgs& a, bool norm, int row_token,
                                        int j) {
    if (norm) {
      double s = 0.0;
#pragma unroll
      for (int l = 0; l < 8; ++l) s = __builtin_fma((double)v[l], (double)v[l], s);
      s = wave_sum<NB>(s);
      // 1 / sqrt(mean + eps) in fp64: two Newton steps from the hardware's reciprocal root
      const double x = s * (1.0 / (8 * NB)) + a.eps;
      // (which is right by itself where the mean is infinite or 0)
      double y = __builtin_amdgcn_rsq(x);
      if (x > 0.0 && x < INFINITY) {
        y = __builtin_fma(0.5 * y, __builtin_fma(-x * y, y, 1.0), y);
        y = __builtin_fma(0.5 * y, __builtin_fma(-x * y, y, 1.0), y);
      }
      const float f = (float)y;
#pragma unroll
      for (int l = 0; l < 8; ++l) v[l] = (v[l] * f) * w[l];
    }
    if (a.rot) {
      const int rb = a.rot >> 3, half = rb >> 1;      // blocks that are turned
      const bool halves = a.pairs == NQ_PAIRS_HALVES, second = halves && j >= half;
      if (__any(row_token != token)) {
        token = row_token;
        int pos = a.positions[token];
        pos = pos < 0 ? 0 : (pos >= a.table_rows ? a.table_rows - 1 : pos);
        if (j < rb) {
          const int64_t at = (int64_t)pos * (a.rot >> 1);
          if (halves) {
            const int64_t i = at + 8 * (second ? j - half : j);
            load8(a.cos + i, c);
            load8(a.sin + i, n);
#pragma unroll
            for (int l = 0; l < 8; ++l) n[l] = second ? n[l] : -n[l];
          } else {
            const f32x4 x = *reinterpret_cast<const f32x4*>(a.cos + at + 4 * j);
            const f32x4 y = *reinterpret_cast<const f32x4*>(a.sin + at + 4 * j);
#pragma unroll
            for (int l = 0; l < 4; ++l) {
              c[2 * l] = c[2 * l + 1] = x[l];
              n[2 * l] = -y[l];
              n[2 * l + 1] = y[l];
            }
          }
        }
      }
      // every entry becomes itself times the cosine plus its partner times the signed sine
      float p[8];
      if (halves) {
        const int other = j < rb ? (second ? j - half : j + half) : j;
        const int src = (int)(threadIdx.x & (64 - NB)) | lane_of_block(other);
#pragma unroll
        for (int l = 0; l < 8; ++l) p[l] = __shfl(v[l], src, 64);
      } else {
#pragma unroll
        for (int l = 0; l < 8; ++l) p[l] = v[l ^ 1];
      }
      if (j < rb) {
#pragma unroll
        for (int l = 0; l < 8; ++l) v[l] = v[l] * c[l] + p[l] * n[l];
      }
    }
    if (a.hadamard) hadamard<NB>(v, j, a.rot_s);
  }
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) |
         (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16;
}

template <typename T>
__device__ __forceinline__ void load_row(const KVRows& x, int token, int head, int j, RawBlock<T>& raw) {
  load_raw<T, false>(reinterpret_cast<const T*>(x.data) + token * x.token_stride +
                         head * x.head_stride + 8 * j, raw);
}

// PASSES passes of 64 / NB query rows from row `first` on, for one wave.
template <typename T, int NB, int PASSES>
__device__ __forceinline__ void query_rows(const KVAppendArgs& a, uint32_t first) {
  constexpr int R = 64 / NB;
  const int lane = (int)threadIdx.x & 63, j = block_of_lane(lane % NB);
  const uint32_t rows = (uint32_t)a.tokens * a.by_q.n;
  RowSteps<NB> steps;
  steps.start(a, a.q_norm, j);
  uint32_t row = first + lane / NB;
  RawBlock<T> ahead;
  int token = 0, head = 0;
  auto fetch = [&]() {
    if (row >= rows) return;
    token = (int)(((uint64_t)row * a.by_q.magic) >> a.by_q.shift);
    head = (int)(row - (uint32_t)token * a.by_q.n);
    load_row<T>(a.q, token, head, j, ahead);
  };
  fetch();
#pragma unroll 1
  for (int i = 0; i < PASSES; ++i) {
    if (row >= rows) break;                       // whole rows of lanes
    float v[8];
    unpack_raw<T>(ahead, v);
    const int now = token;
    const int64_t o = token * a.out.token_stride + head * a.out.head_stride + 8 * j;
    row += R;
    if (i + 1 < PASSES) fetch();                  // the next pass's, while this one is worked on
    steps.apply(v, a, a.q_norm != nullptr, now, j);
    if (a.out_dtype == NQ_F32) {
      f32x4* p = reinterpret_cast<f32x4*>((float*)a.out.data + o);
      p[0] = f32x4{v[0], v[1], v[2], v[3]};
      p[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      u32x4 w;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        w[u] = a.out_dtype == NQ_F16 ? pack_f16(v[2 * u], v[2 * u + 1])
                                     : pack_bf16(v[2 * u], v[2 * u + 1]);
      *reinterpret_cast<u32x4*>((uint16_t*)a.out.data + o) = w;
    }
  }
}

// Queries in a launch of their own, for many rows: four waves a workgroup and no LDS, so that
// twice as many waves are resident as beside the encoder's.
constexpr int kQueryPasses = 16;
template <typename T, int NB>
__global__ __launch_bounds__(256) void kv_query_kernel(KVAppendArgs a) {
  const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6);
  query_rows<T, NB, kQueryPasses>(a, wave * (uint32_t)(64 / NB * kQueryPasses));
}

// A workgroup is one wave and takes BPT passes of 64 / NB rows of one kind: keys first, then
// values, then queries.  Rows of keys and values that their first beta does not settle are
// staged in LDS and finished together after the passes (see encode_wave_kernel).
template <typename T, int NB, int BPT>
__global__ __launch_bounds__(64) void kv_append_kernel(KVAppendArgs a, int wgs_kv) {
  constexpr int R = 64 / NB, RW = R * BPT, SLOTS = 64 * BPT;
  __shared__ __attribute__((aligned(16))) float staged[SLOTS][8];
  __shared__ uint16_t queue[SLOTS];               // slot << 2 | t
  __shared__ uint8_t tsl[SLOTS];
  __shared__ float crow[RW][4];
  __shared__ __attribute__((aligned(16))) float chi[RW][4];
  __shared__ int64_t at[RW];                      // row of the pool, -1: none

  const int lane = (int)threadIdx.x, l = lane % NB, j = block_of_lane(l);
  const int kind = (int)blockIdx.x < wgs_kv ? 0 : ((int)blockIdx.x < 2 * wgs_kv ? 1 : 2);
  const int wg = (int)blockIdx.x - kind * wgs_kv;
  if (kind == 2) {
    query_rows<T, NB, BPT>(a, (uint32_t)wg * RW);
    return;
  }

  const bool keys = kind == 0;
  EncodeArgs e;     // the fields the encoder's pieces read
  e.q = keys ? a.ck.q : a.cv.q;
  e.k = keys ? a.ck.k : a.cv.k;
  e.rq = keys ? a.ck.rq : a.cv.rq;
  e.m2q = keys ? a.ck.m2q : a.cv.m2q;
  e.mq = keys ? a.ck.mq : a.cv.mq;
  e.decoder = keys ? a.ck.decoder : a.cv.decoder;
  const int t = l & 3;   // the beta whose multiplier and limits this lane finds
  auto beta_of = [&](int i) {
    const double k = i == 0 ? a.ck.beta[0] : (i == 1 ? a.ck.beta[1] : (i == 2 ? a.ck.beta[2] : a.ck.beta[3]));
    const double v = i == 0 ? a.cv.beta[0] : (i == 1 ? a.cv.beta[1] : (i == 2 ? a.cv.beta[2] : a.cv.beta[3]));
    return keys ? k : v;
  };
  const double beta_t = beta_of(t), beta_last = beta_of(e.k - 1);
  const KVPool pool = keys ? a.pk : a.pv;
  const uint32_t rows = (uint32_t)a.tokens * a.by_kv.n;
  constexpr double n = 8 * NB;
  RowSteps<NB> steps;
  steps.start(a, keys ? a.k_norm : nullptr, j);
  int qn = 0;
#pragma unroll 1
  for (int i = 0; i < BPT; ++i) {
    const int rw = i * R + lane / NB, sl = i * 64 + lane;
    const uint32_t row = (uint32_t)wg * RW + rw;
    bool valid = row < rows;
    int64_t prow = -1;
    float v[8] = {};
    if (valid) {
      const int token = (int)(((uint64_t)row * a.by_kv.magic) >> a.by_kv.shift);
      const int head = (int)(row - (uint32_t)token * a.by_kv.n);
      const int64_t slot = a.slots[token];
      valid = slot >= 0 && slot < a.limit;
      if (valid) {
        const int64_t page = slot >> a.page_shift;
        prow = ((page * a.heads + head) << a.page_shift) | (slot & ((1ll << a.page_shift) - 1));
      }
      RawBlock<T> raw;
      load_row<T>(keys ? a.k : a.v, token, head, j, raw);
      unpack_raw<T>(raw, v);
      if (keys) steps.apply(v, a, a.k_norm != nullptr, token, j);
    }
    // the row scale, the multiplier and the limits of beta t, one t a lane of every four
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) s = __builtin_fma((double)v[u], (double)v[u], s);
    s = wave_sum<NB>(s);
    bool sure;
    float r = rms_candidate(s, n, 1.0 / n, sure);
    if (!sure) {
      double hi = 0.0, lo = 0.0;
#pragma unroll
      for (int u = 0; u < 8; ++u) dd_add_square(hi, lo, v[u]);
#pragma unroll
      for (int m = 1; m < NB; m <<= 1) {
        const double oh = __shfl_xor(hi, m, 64), ol = __shfl_xor(lo, m, 64);
        double sd, ed;
        two_sum(hi, oh, sd, ed);
        hi = sd;
        lo = lo + ol + ed;
      }
      double sd, ed;
      two_sum(hi, lo, sd, ed);
      r = exact_rms(sd, ed, n, r);
    }
    const bool coded = valid && (r > 0.0f) && isfinite(r);
    {
      const double rb = (double)r * beta_t;
      float hi = INFINITY;
      if (t == 3 || t < e.k - 1)
        hi = row_limit(t == 3 ? kBytesFactor : skip_factor(e.q, e.decoder),
                       t == 3 ? (double)r * beta_last : rb);
      if (l < 4) {
        crow[rw][t] = coded ? (float)(1.0 / rb) : 0.0f;
        chi[rw][t] = hi;
        if (t == 0) at[rw] = prow;
      }
    }
    if (valid && l == 0) pool.scales[prow] = r;
    __syncthreads();   // one wave: the LDS of its rows

    bool queued = false;
    int start = 0, t0 = 0;
    uint32_t word = 0u;
    if (coded) {
      const float mx = e.decoder ? m_stat(v) : root_bound_f(v);
      const f32x4 hi = *reinterpret_cast<const f32x4*>(chi[rw]);
      t0 = mx > hi.x ? (mx > hi.y ? (mx > hi.z ? 3 : 2) : 1) : 0;
      E8Bytes P;
      const Verdict vd = eval_bytes<false>(v, crow[rw][t0], t0, e, P, word);
      const bool past = mx > hi.w;
      queued = vd != KEEP || past;
      start = t0 + (vd == NEXT && !past ? 1 : 0);
    }
    const uint64_t mask = __ballot(queued);
    if (queued) {
      *reinterpret_cast<f32x4*>(&staged[sl][0]) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(&staged[sl][4]) = f32x4{v[4], v[5], v[6], v[7]};
      queue[qn + __popcll(mask & ((1ull << lane) - 1ull))] = (uint16_t)((sl << 2) | start);
    } else {
      if (valid) pool.codes[prow * NB + j] = word;
      tsl[sl] = (uint8_t)t0;
    }
    qn += __popcll(mask);
  }
  __syncthreads();

  // the queued blocks, one beta a round, compacted in place (entries already read)
#pragma unroll 1
  while (qn > 0) {
    int nn = 0;
#pragma unroll 1
    for (int base = 0; base < qn; base += 64) {
      const int idx = base + lane;
      bool more = false;
      uint32_t next = 0;
      if (idx < qn) {
        const uint32_t ent = queue[idx];
        const int sl = (int)(ent >> 2), t = (int)(ent & 3u);
        const int ll = sl & 63, rw = (sl >> 6) * R + ll / NB;
        float v[8];
        load8(&staged[sl][0], v);
        const float ct = crow[rw][t];
        const float vmax = max3_abs(max3_abs(v[0], v[1], v[2]), max3_abs(v[3], v[4], v[5]),
                                    max3_abs(v[6], v[7], v[7]));
        E8Bytes Pb;
        uint32_t word = 0u;
        const Verdict vd = vmax <= chi[rw][3] ? eval_bytes<true>(v, ct, t, e, Pb, word) : EXACT;
        bool done = vd == KEEP;
        if (vd == EXACT) {
          int P[8];
          done = eval_exact(v, ct, t, e, P);
          if (done) word = encode_codes(P, e.q, e.rq, e.mq);
        }
        if (done) {
          pool.codes[at[rw] * NB + block_of_lane(ll % NB)] = word;
          tsl[sl] = (uint8_t)t;
        }
        more = !done;
        next = ((uint32_t)sl << 2) | (uint32_t)(t + 1);
      }
      const uint64_t mask = __ballot(more);
      if (more) queue[nn + __popcll(mask & ((1ull << lane) - 1ull))] = (uint16_t)next;
      nn += __popcll(mask);
    }
    __syncthreads();
    qn = nn;
  }

  // beta words: the 16 (or 8) two-bit indices of a group of lanes
  constexpr int NBW = (NB + 15) / 16;
#pragma unroll
  for (int i = 0; i < BPT; ++i) {
    const int rw = i * R + lane / NB;
    const int64_t prow = at[rw];
    uint32_t bits = (uint32_t)tsl[i * 64 + lane] << (2 * (j & 15));
    bits |= dpp_across<1>(bits);
    bits |= dpp_across<2>(bits);
    bits |= dpp_across<4>(bits);
    if constexpr (NB > 8) bits |= dpp_across<8>(bits);
    if (prow >= 0 && (l & 15) == 0) pool.beta[prow * NBW + (l >> 4)] = bits;
  }
}

template <typename T, int NB, int BPT>
hipError_t launch(const KVAppendArgs& a, bool apart, hipStream_t st) {
  constexpr int64_t RW = 64 / NB * BPT;
  const int64_t kv = ((int64_t)a.tokens * a.heads + RW - 1) / RW;
  const int64_t q = apart ? 0 : ((int64_t)a.tokens * a.q_heads + RW - 1) / RW;
  hipLaunchKernelGGL((kv_append_kernel<T, NB, BPT>), dim3((unsigned)(2 * kv + q)), dim3(64), 0, st, a,
                     (int)kv);
  if (apart) {
    constexpr int64_t QW = 4 * (64 / NB) * kQueryPasses;
    const int64_t wgs = ((int64_t)a.tokens * a.q_heads + QW - 1) / QW;
    hipLaunchKernelGGL((kv_query_kernel<T, NB>), dim3((unsigned)wgs), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

template <typename T, int NB>
hipError_t launch_dim(const KVAppendArgs& a, hipStream_t st) {
  // Four passes a wave fill the lanes that finish the queue, once there are waves for every
  // SIMD.  Queries of many million blocks get a launch of their own, at the rate of memory
  // (16384 tokens of 64 heads: 206-226 us, 236 in one launch); fewer run better behind the
  // encoder's waves (4096 tokens of 32 heads: 34 us, 46 apart).
  const bool many = (int64_t)a.tokens * a.heads * NB >= (int64_t)4 * 1024 * 64;
  const bool apart = (int64_t)a.tokens * a.q_heads * NB >= (int64_t)1 << 23;
  return many ? launch<T, NB, 4>(a, apart, st) : launch<T, NB, 1>(a, apart, st);
}

template <typename T>
hipError_t launch_type(const KVAppendArgs& a, int dim, hipStream_t st) {
  switch (dim) {
    case 64: return launch_dim<T, 8>(a, st);
    case 128: return launch_dim<T, 16>(a, st);
    default: return launch_dim<T, 32>(a, st);
  }
}

}  // namespace

hipError_t launch_kv_append(const KVAppendArgs& a, int dtype, int dim, hipStream_t st) {
  switch (dtype) {
    case NQ_F32: return launch_type<float>(a, dim, st);
    case NQ_F16: return launch_type<_Float16>(a, dim, st);
    default: return launch_type<uint16_t>(a, dim, st);
  }
}

}  // namespace nq
