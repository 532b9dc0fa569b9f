// Attention of few query rows over a coded KV cache (nq_attend), split over the cache's length.
//
// A workgroup takes one KV head of one sequence, a block of its query rows (the queries of the
// heads that share the KV head) and a chunk of the tokens they see.  Its four waves step
// through the chunk in turn, 32 tokens a step (16 where the call has few), each with its own
// references and sums:
//   * the scores are S^T = K Q^T on 16x16x32 fp16 matrix instructions.  Lane l holds the blocks
//     of token l % 16 in the A operand, so a lane decodes its code words (16 bytes of a row)
//     straight into the operand; the order of the entries along the contraction is that of the
//     lanes' blocks, and Q's operand is laid out to match;
//   * S^T leaves four tokens of one query row in each lane, which is what the B operand of
//     O^T += V^T P^T holds (in an order of the tokens of its own), so the weights stay in
//     registers; the references of the sums (RowSum) move seldom, and only then is a maximum
//     taken across lanes;
//   * V's blocks are decoded into LDS and read back transposed (ds_read_b64_tr_b16).
// The decoded values are integers m X2 / 8, exact in fp16; the rows' scales multiply the scores
// and the weights in fp32.  Queries in 16 bits are exact in one fp16 operand (scaled by a power
// of two), fp32 ones and the weights are taken as the sum of two (22 bits).
//
// The waves' results are joined in LDS, the chunks' by join_kernel, in a fixed order.
//
// What bounds it: vector instructions, about 2040 a step of 32 tokens and wave, of which 16 blocks a
// lane take 105 each; 0.98 a clock of a busy CU.  131072 tokens of 8 KV heads: 123 us (1.2 TB/s of
// codes, a quarter of what a copy reaches); 64 ragged sequences of up to 8192: 290-298 us.  Three
// waves a SIMD without scratch beat four with it (250 against 280 us at 32 x 8192 tokens).
#include <type_traits>

#include "nq_attend.hpp"
#include "nq_attend_join.hpp"

namespace nq {
namespace {

constexpr int kWaves = 4;

template <int DIM>
struct Shape {
  static constexpr int NB = DIM / 8;           // blocks of a row
  static constexpr int NBL = NB / 4;           // of a lane: steps of the contraction over entries
  static constexpr int DT = DIM / 16;          // 16-entry tiles of an output row
  static constexpr int PITCH = DIM + 8;        // halves of a row of decoded V in LDS
  static constexpr int OP = DIM + 4;           // floats of an output row in LDS
  static constexpr int VBYTES = 32 * PITCH * 2;
  static constexpr int OBYTES = 16 * OP * 4;
  static constexpr int LDS = kWaves * (VBYTES > OBYTES ? VBYTES : OBYTES);
};

// What a lane needs of a step's U x 16 tokens of one pool: its blocks, and the scales of the
// tokens whose scores it gets (four of each 16).
template <int NBL, int U>
struct StepWords {
  Words<NBL> w[U];
  f32x4 scales[U];
};

// A step's tiles: their first tokens, their rows in the pools, and whether they count.
template <int U>
struct StepRows {
  int tok[U];
  int64_t row[U];
  bool ok[U];
};
template <int U>
__device__ __forceinline__ StepRows<U> rows_of(const AttendArgs& a, const Tiles& tiles, int b,
                                               int head, int step) {
  StepRows<U> r;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool there = U * step + u < tiles.count;
    r.tok[u] = 16 * tiles.tile(there ? U * step + u : U * step);
    r.row[u] = tile_row(a, b, head, r.tok[u], r.ok[u]);
    r.ok[u] = r.ok[u] & there;
  }
  return r;
}
template <int NBL, int U>
__device__ __forceinline__ void load_step(const AttendPool& p, const StepRows<U>& r, int t, int g,
                                          StepWords<NBL, U>& s) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    s.w[u] = load_words<NBL>(p, r.row[u] + t, g);
    s.scales[u] = *reinterpret_cast<const f32x4*>(p.scales + r.row[u] + 4 * g);
  }
}

// RT: 16-row tiles of the row block.  M: NestQuantM's decoder.  TERMS: fp16 terms of a query.
// U: 16-token tiles of a step, two, or one where a call has few tiles (attend_plan).
template <int DIM, int RT, bool M, int TERMS, int U>
__global__ __launch_bounds__(64 * kWaves)
__attribute__((amdgpu_waves_per_eu(DIM <= 128 && RT == 1 && TERMS == 1 ? 3 : (DIM <= 128 ? 2 : 1)))) void attend_kernel(AttendArgs a) {
  using S = Shape<DIM>;
  constexpr int NBL = S::NBL, DT = S::DT;
  using Weights = typename std::conditional<U == 2, h8, h4>::type;   // a lane's weights of a step
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ float wave_m[kWaves][16 * RT], wave_l[kWaves][16 * RT];

  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int lane = (int)threadIdx.x & 63, t = lane & 15, g = lane >> 4;
  const Place at = place_of(a, blockIdx.x);
  const int head = at.head, b = at.b, rb = at.part % a.blocks, chunk = at.part / a.blocks;
  const Sequence sq = sequence_of(a, b);
  const int group = (int)a.by_group.n;
  const RowBlock blk = row_block<16 * RT>(a, sq, rb);
  const int r0 = blk.r0, rows = blk.rows;
  if (rows <= 0) return;
  const Tiles tiles = tiles_of<4>(a, blk.p_lo, blk.p_hi, sq.end);
  const int steps = (tiles.count + U - 1) / U;
  const int s_end = steps < (chunk + 1) * a.steps ? steps : (chunk + 1) * a.steps;
  if (chunk > 0 && chunk * a.steps >= steps) return;

  // the query rows of this lane's column, as operands, and their positions
  h8 qop[RT][TERMS][NBL];
  float q_scale[RT];
  Range range[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + 16 * rt + t;
    const bool there = 16 * rt + t < rows;
    const int i = query_of(a, there ? r : r0), hq = (there ? r : r0) - i * group;
    const int64_t base = (int64_t)(sq.first + i) * a.q.token_stride +
                         (int64_t)(head * group + hq) * a.q.head_stride + 8 * NBL * g;
    range[rt] = range_of(a, sq.shift + i, sq.end);
    float x[NBL][8], mx = 0.0f;
    load_query<TERMS == 2, NBL, 8>(a.q.data, a.dtype, base, x);   // past the last row: the first
#pragma unroll
    for (int s = 0; s < NBL; ++s)
#pragma unroll
      for (int l = 0; l < 8; ++l) mx = fmaxf(mx, fabsf(x[s][l]));
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    // a power of two brings the row's largest entry to [2^14, 2^15)
    const int e = row_exponent(mx);
    q_scale[rt] = a.k_scale * __builtin_ldexpf(1.0f, e - 14);
#pragma unroll
    for (int s = 0; s < NBL; ++s)
#pragma unroll
      for (int l = 0; l < 8; ++l) {
        const float v = settled(__builtin_ldexpf(x[s][l], 14 - e));
        const _Float16 h = (_Float16)v;
        qop[rt][0][s][l] = h;
        if constexpr (TERMS == 2) qop[rt][1][s][l] = (_Float16)(v - (float)h);
      }
  }

  f32x4 o[RT][DT] = {};
  RowSum sum[RT];
  _Float16* vt = reinterpret_cast<_Float16*>(lds + wave * S::VBYTES);

  // The code words are loaded ahead: a step's values while its keys are decoded, the next
  // step's keys while its values are.
  StepRows<U> cur;
  StepWords<NBL, U> kw, vw;
  int st = chunk * a.steps + wave;
  if (st < s_end) {
    cur = rows_of<U>(a, tiles, b, head, st);
    load_step<NBL, U>(a.k, cur, t, g, kw);
  }
  for (; st < s_end; st += kWaves) {
    load_step<NBL, U>(a.v, cur, t, g, vw);
    const bool more = st + kWaves < s_end;
    const StepRows<U> next = rows_of<U>(a, tiles, b, head, more ? st + kWaves : st);
    // scores
    f32x4 acc[RT][U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int s = 0; s < NBL; ++s) {
        const h8 kop = decode_f16<M>(kw.w[u].w[s], (kw.w[u].beta >> (2 * s)) & 3u, a.ck);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int x = 0; x < TERMS; ++x)
            acc[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kop, qop[rt][x][s], acc[rt][u], 0, 0, 0);
      }
    }
    f32x4 ks[U];
#pragma unroll
    for (int u = 0; u < U; ++u) ks[u] = kw.scales[u];
    if (more) load_step<NBL, U>(a.k, next, t, g, kw);

    // a bound of the scales of this lane's tokens (2^lv), seen or not
    float lv = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) lv = fmaxf(lv, finite_size(vw.scales[u][i]));
    lv = __builtin_amdgcn_logf(lv);

    Weights pop[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float sc[U][4], mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool see = cur.ok[u] & range[rt].sees(cur.tok[u] + 4 * g + i);
          const float v = acc[rt][u][i] * (ks[u][i] * q_scale[rt]);
          sc[u][i] = see ? v : -INFINITY;
          mx = fmaxf(mx, sc[u][i]);
        }
      // new references only where these tokens might pass the present ones
      if (__any(sum[rt].passed(mx, lv))) {
        float both = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            both = fmaxf(both, sc[u][i] + __builtin_amdgcn_logf(finite_size(vw.scales[u][i])));
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        both = fmaxf(both, __shfl_xor(both, 16, 64));
        both = fmaxf(both, __shfl_xor(both, 32, 64));
        const float f = sum[rt].raise(mx, both);
        if (__any(f != 1.0f)) {
#pragma unroll
          for (int d = 0; d < DT; ++d) o[rt][d] *= f;
        }
      }
      float e = 0.0f, w[U][4];
      if (!sum[rt].wide) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(sc[u][i] - sum[rt].ref);
            e += p;
            w[u][i] = p * vw.scales[u][i];
          }
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e += sum[rt].term(sc[u][i] - sum[rt].ref, sc[u][i] - sum[rt].m, vw.scales[u][i], w[u][i]);
          }
      }
      sum[rt].add(e);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // a token that is not seen has weight 0, whatever its scale
          const float x = settled(sc[u][i] == -INFINITY ? 0.0f : w[u][i]);
          const _Float16 h = (_Float16)x;
          pop[rt][0][4 * u + i] = h;
          pop[rt][1][4 * u + i] = (_Float16)(x - (float)h);
        }
    }
    // V: decoded rows into LDS, columns of four tokens back
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < NBL; ++s) {
        const h8 x = decode_f16<M>(vw.w[u].w[s], (vw.w[u].beta >> (2 * s)) & 3u, a.cv);
        *reinterpret_cast<h8*>(vt + (16 * u + t) * S::PITCH + 8 * (NBL * g + s)) = x;
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const _Float16* from = vt + (4 * g + (t >> 2)) * S::PITCH + 4 * (t & 3);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const h4 lo = read_transposed(from + 16 * d);
      if constexpr (U == 2) {
        const h4 hi = read_transposed(from + 16 * S::PITCH + 16 * d);
        const h8 vop = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vop, pop[rt][0], o[rt][d], 0, 0, 0);
          o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vop, pop[rt][1], o[rt][d], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x16f16(lo, pop[rt][0], o[rt][d], 0, 0, 0);
          o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x16f16(lo, pop[rt][1], o[rt][d], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
    cur = next;
  }

  // join the waves
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt].l += __shfl_xor(sum[rt].l, 16, 64);
    sum[rt].l += __shfl_xor(sum[rt].l, 32, 64);
    if (g == 0) {
      wave_m[wave][16 * rt + t] = sum[rt].m;
      wave_l[wave][16 * rt + t] = sum[rt].l;
    }
  }
  float* ob = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    __syncthreads();
    float mm = wave_m[0][16 * rt + t];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, wave_m[w][16 * rt + t]);
    // o holds the sums over V relative to 2^ref
    const float f = half_power(sum[rt].ref - mm);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      *reinterpret_cast<f32x4*>(ob + (wave * 16 + t) * S::OP + 16 * d + 4 * g) = (o[rt][d] * f) * (f * a.v_scale);
    __syncthreads();
    for (int x = (int)threadIdx.x; x < 16 * (DIM / 4); x += 64 * kWaves) {
      const int row = x / (DIM / 4), c = x % (DIM / 4), r = 16 * rt + row;
      if (r >= rows) continue;
      f32x4 all = {};
      float big = -INFINITY, total = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        all += *reinterpret_cast<const f32x4*>(ob + (w * 16 + row) * S::OP + 4 * c);
        big = fmaxf(big, wave_m[w][r]);
      }
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        total += wave_l[w][r] * __builtin_amdgcn_exp2f(wave_m[w][r] - big);
      const int i = query_of(a, r0 + r), hq = head * group + r0 + r - i * group;
      const int64_t token = sq.first + i;
      if (a.chunks == 1) {
        store_out(a.out, a.dtype, token * a.out_token + hq * a.out_head + 4 * c, all * inverse_sum(total));
        if (a.lse && c == 0) a.lse[token * a.q_heads + hq] = log_sum(big, total);
      } else {
        float* p = partial(a, b, head, rb, r, chunk, DIM);
        *reinterpret_cast<f32x4*>(p + 4 + 4 * c) = all;
        if (c == 0) {
          p[0] = big;
          p[1] = total;
        }
      }
    }
  }
}

template <int DIM, int RT, bool M, int U>
hipError_t launch(const AttendArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.chunks * a.blocks * a.heads * a.seqs));
  constexpr int bytes = Shape<DIM>::LDS;
  if (a.dtype == NQ_F32) {
    hipLaunchKernelGGL((attend_kernel<DIM, RT, M, 2, U>), grid, dim3(64 * kWaves), bytes, st, a);
  } else {
    hipLaunchKernelGGL((attend_kernel<DIM, RT, M, 1, U>), grid, dim3(64 * kWaves), bytes, st, a);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && a.chunks > 1 ? launch_join<DIM, 16 * RT, 4, U>(a, st) : e;
}

template <int DIM, int RT, int U>
hipError_t attributes() {
  constexpr int bytes = Shape<DIM>::LDS;
  for (const void* f : {(const void*)attend_kernel<DIM, RT, false, 1, U>, (const void*)attend_kernel<DIM, RT, false, 2, U>,
                        (const void*)attend_kernel<DIM, RT, true, 1, U>, (const void*)attend_kernel<DIM, RT, true, 2, U>}) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

// The forms that a plan may ask for (attend_plan): dim, 16-row tiles, tiles of tokens a step.
#define NQ_FORMS(X)                                                             \
  X(64, 1, 1) X(64, 1, 2) X(64, 2, 2) X(128, 1, 1) X(128, 1, 2) X(128, 2, 2)    \
  X(256, 1, 1) X(256, 1, 2)

hipError_t attend_set_attributes() {
  hipError_t e = hipSuccess;
#define NQ_SET(D, R, U) \
  if (e == hipSuccess) e = attributes<D, R, U>();
  NQ_FORMS(NQ_SET)
#undef NQ_SET
  return e;
}

hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, int dim, int decoder,
                         hipStream_t st) {
#define NQ_GO(D, R, U)                                  \
  if (dim == D && p.tiles == R && p.units == U)         \
    return decoder ? launch<D, R, true, U>(a, st) : launch<D, R, false, U>(a, st);
  NQ_FORMS(NQ_GO)
#undef NQ_GO
  return hipErrorInvalidValue;
}

}  // namespace nq
