// Attention of many query rows over a coded KV cache (nq_attend): prompts and chunks of them.
//
// A code word takes about 110 vector instructions to decode, so every token that the call's
// queries see is decoded once, by unpack_kernel, into the workspace, in records of 64 tokens of
// one KV head: K and V as the fp16 integers m X2 / 8 (exact) in the order in which the matrix
// instructions' operands lie in registers, the rows' scales, and which tokens count.
//
// prompt_kernel gives a workgroup of four waves 128 query rows of a KV head (its group's heads
// side by side), 32 rows a wave, and runs over the records that its rows see: the records come
// into LDS by direct loads, one ahead of the one in use, and every operand is one 16-byte LDS read a
// lane without bank conflicts.  Per record and wave, on 32x32x16 matrix instructions:
//   S^T = K Q^T, 2 x DIM / 16 of them;  O^T += V^T P^T, 8 x DIM / 32 (twice as many of the first
//   for fp32 queries).
// S^T leaves 16 tokens of one query row in each lane, in the order that the B operand of the
// second product takes (V's operands are laid out to match), so the weights never leave the
// lane.  The keys' scales multiply the scores, the values' the weights, in fp32.
//
// The weights are the sum of two fp16 numbers (22 bits) whatever the queries' type: one number, 11
// bits, is no more than fp16 outputs keep, and a call of 64 rows or fewer keeps 22.  The second
// term's matrix instructions make 8192 queries 620 -> 800 us.
//
// What bounds it: per 64 tokens and 32 rows a wave issues 48 matrix instructions (1536 clocks of its
// SIMD at DIM = 128), about 220 vector instructions and 32 exponentials (1400) and reads 32 KiB
// of LDS; two waves a SIMD overlap them in part.  8192 queries of 32 heads: 800-823 us, 668-687
// TFLOP/s; 2048: 83-91 us, where one round of workgroups with 1 to 32 records each is the limit.
#include <type_traits>

#include "nq_attend.hpp"
#include "nq_attend_join.hpp"

namespace nq {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kRows = 32 * kWaves;

// A record: K's operands, V's, 64 scales of the keys, 64 of the values, the bits of the tokens that
// count, the logarithm of the values' largest finite scale, and whether all of them are finite.
template <int DIM>
struct Record {
  static constexpr int V = DIM * 128, KS = DIM * 256, VS = KS + 256, BITS = VS + 256, TOP = BITS + 8, FINITE = TOP + 4;
  static constexpr int BYTES = DIM * 256 + 1024;
};

template <int DIM, bool M>
__global__ __launch_bounds__(256) void unpack_kernel(AttendArgs a) {
  using R = Record<DIM>;
  constexpr int NBL = DIM / 32, PITCH = DIM + 8;
  __shared__ __attribute__((aligned(16))) _Float16 vt[64 * PITCH];
  const Place at = place_of(a, blockIdx.x);
  const int u = at.part, head = at.head, b = at.b;
  const Sequence sq = sequence_of(a, b);
  if (sq.queries == 0) return;
  const Tiles tiles = tiles_of<6>(a, sq.shift, sq.shift + sq.queries - 1, sq.end);
  if (u >= tiles.count) return;
  unsigned char* rec = a.records + (((int64_t)b * a.heads + head) * a.groups + u) * R::BYTES;
  const int lane = (int)threadIdx.x & 63;
  const int g = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // lane: token; wave: a quarter of the row's blocks
  const int token = 64 * tiles.tile(u) + lane;
  const bool in = token < sq.end;
  bool ok;
  const int64_t row = tile_row(a, b, head, in ? token : 0, ok);
  ok = ok && in;
  const Words<NBL> kw = load_words<NBL>(a.k, row, g), vw = load_words<NBL>(a.v, row, g);
#pragma unroll
  for (int s = 0; s < NBL; ++s) {
    const int j = NBL * g + s;
    const h8 k = decode_f16<M>(kw.w[s], (kw.beta >> (2 * s)) & 3u, a.ck);
    const h8 v = decode_f16<M>(vw.w[s], (vw.beta >> (2 * s)) & 3u, a.cv);
    // K: tile of 32 tokens, step of 16 entries, half of it, token
    *reinterpret_cast<h8*>(rec + ((((lane >> 5) * (DIM / 16) + (j >> 1)) * 64 + (j & 1) * 32 + (lane & 31)) << 4)) = k;
    *reinterpret_cast<h8*>(vt + lane * PITCH + 8 * j) = v;
  }
  if (g == 0) {
    const float ks = a.k.scales[row], vs = a.v.scales[row];
    float most = ok ? finite_size(vs) : 0.0f;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    reinterpret_cast<float*>(rec + R::KS)[lane] = ok ? ks : 0.0f;
    reinterpret_cast<float*>(rec + R::VS)[lane] = ok ? vs : 0.0f;
    const uint64_t bits = __ballot(ok), odd = __ballot(ok && !isfinite(vs));
    if (lane == 0) {
      *reinterpret_cast<uint64_t*>(rec + R::BITS) = bits;
      *reinterpret_cast<float*>(rec + R::TOP) = __builtin_amdgcn_logf(most);
      *reinterpret_cast<uint32_t*>(rec + R::FINITE) = odd == 0;
    }
  }
  __syncthreads();
  // V^T: tile of 32 entries, step of 16 tokens; lane l holds entry l % 32 and, with h = l / 32,
  // tokens 4 h .. + 3 and 8 + 4 h .. + 3 of the step (wave g: step g)
  const int q = lane >> 4, i = lane & 15;
  const _Float16* from = vt + (16 * g + 4 * (q >> 1) + (i >> 2)) * PITCH + 16 * (q & 1) + 4 * (i & 3);
#pragma unroll
  for (int d = 0; d < DIM / 32; ++d) {
    const h4 lo = read_transposed(from + 32 * d), hi = read_transposed(from + 8 * PITCH + 32 * d);
    *reinterpret_cast<h8*>(rec + R::V + (((d * 4 + g) * 64 + lane) << 4)) =
        h8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  }
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// TERMS: fp16 terms of the queries (the weights have two).
template <int DIM, int TERMS>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(DIM <= 128 && TERMS == 1 ? 2 : 1))) void prompt_kernel(AttendArgs a) {
  using R = Record<DIM>;
  constexpr int KS = DIM / 16, DT = DIM / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  typedef __attribute__((address_space(3))) void lds_void;

  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int lane = (int)threadIdx.x & 63, t = lane & 31, h = lane >> 5;
  // The last rows of a prompt see the most tokens: they start first.  A grid that fits the chip at
  // once, two workgroups a CU, has its second half in the other order, so that a CU's two
  // share the work out evenly.
  const Place at = place_of(a, blockIdx.x);
  const int head = at.head, b = at.b, chunk = at.part % a.chunks;
  int rb = at.part / a.chunks;
  rb = a.mirror && rb >= (a.blocks >> 1) ? rb - (a.blocks >> 1) : a.blocks - 1 - rb;
  const Sequence sq = sequence_of(a, b);
  const int group = (int)a.by_group.n;
  const RowBlock blk = row_block<kRows>(a, sq, rb);
  if (blk.rows <= 0) return;
  const Tiles all = tiles_of<6>(a, sq.shift, sq.shift + sq.queries - 1, sq.end);
  const Tiles tiles = tiles_of<6>(a, blk.p_lo, blk.p_hi, sq.end);
  const int first = chunk * a.steps;
  const int last = tiles.count < first + a.steps ? tiles.count : first + a.steps;
  if (chunk > 0 && first >= tiles.count) return;
  const unsigned char* recs = a.records + ((int64_t)b * a.heads + head) * a.groups * R::BYTES;

  // this wave's rows: a lane's column is row r0 + 32 wave + t
  const int mine = blk.rows - 32 * wave;           // of its 32 rows that exist
  const bool there = t < mine;
  const int r = blk.r0 + (there ? 32 * wave + t : 0);
  const int i = query_of(a, r), hq = head * group + r - i * group;
  const Range range = range_of(a, sq.shift + i, sq.end);
  const int w_lo = sq.shift + query_of(a, blk.r0 + (mine > 0 ? 32 * wave : 0));
  const int w_hi = sq.shift + query_of(a, blk.r0 + (mine > 0 ? 32 * wave + (mine < 32 ? mine : 32) - 1 : 0));

  h8 qop[TERMS][KS];
  float q_scale;
  {
    const int64_t base = (int64_t)(sq.first + i) * a.q.token_stride + (int64_t)hq * a.q.head_stride + 8 * h;
    float x[KS][8], mx = 0.0f;
    load_query<TERMS == 2, KS, 16>(a.q.data, a.dtype, base, x);   // past the last row: the first
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int l = 0; l < 8; ++l) mx = fmaxf(mx, fabsf(x[s][l]));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const int e = row_exponent(mx);
    // the scale's size multiplies the scores, its sign the queries; never quite 0, so that the
    // scores of tokens that are not seen stay -infinity
    q_scale = fmaxf(fabsf(a.k_scale) * __builtin_ldexpf(1.0f, e - 14), 0x1p-126f);
    const float sign = a.k_scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int l = 0; l < 8; ++l) {
        const float v = settled(sign * __builtin_ldexpf(x[s][l], 14 - e));
        const _Float16 f = (_Float16)v;
        qop[0][s][l] = f;
        if constexpr (TERMS == 2) qop[1][s][l] = (_Float16)(v - (float)f);
      }
  }

  f32x16 o[DT] = {};
  RowSum sum;

  // a record into buffer `to`: 1 KiB a wave instruction
  auto fetch = [&](int u, int to) {
    const unsigned char* src = recs + (int64_t)all.index(tiles.tile(u)) * R::BYTES + 16 * lane;
    unsigned char* dst = lds + to * R::BYTES;
#pragma unroll
    for (int x = 0; x < DIM / 4; x += kWaves)
      __builtin_amdgcn_global_load_lds((const void*)(src + (x + wave) * 1024),
                                       (lds_void*)(dst + (x + wave) * 1024), 16, 0, 0);
    if (wave == 0)
      __builtin_amdgcn_global_load_lds((const void*)(src + DIM * 256), (lds_void*)(dst + DIM * 256), 16, 0, 0);
  };
  if (first < last) fetch(first, 0);
  for (int u = first; u < last; ++u) {
    const int buf = (u - first) & 1;
    // this record has landed (each wave's share, then everyone's), and no wave reads the
    // other buffer any more: every load and LDS read of this wave is done
    __builtin_amdgcn_s_waitcnt(0x7 << 4);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    if (u + 1 < last) fetch(u + 1, buf ^ 1);
    const unsigned char* rec = lds + buf * R::BYTES;
    const int j0 = 64 * tiles.tile(u);
    if (mine <= 0 || j0 > w_hi || (a.window > 0 && j0 + 63 <= w_lo - a.window && j0 >= a.sinks))
      continue;                                    // nothing for this wave
    const uint64_t bits = *reinterpret_cast<const uint64_t*>(rec + R::BITS);
    const bool whole = bits == ~0ull && j0 + 63 <= w_lo &&
                       (a.window == 0 || j0 > w_hi - a.window || j0 + 63 < a.sinks);

    // all of K's operands on their way before the first is used
    h8 kop[2][KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        kop[x][k] = *reinterpret_cast<const h8*>(rec + (((x * KS + k) * 64 + lane) << 4));
    f32x16 s[2] = {};
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < TERMS; ++y)
          s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kop[x][k], qop[y][k], s[x], 0, 0, 0);
    // the first of V's, read while the weights are formed
    h8 vop[2][4];
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        vop[d][k] = *reinterpret_cast<const h8*>(rec + R::V + (((d * 4 + k) * 64 + lane) << 4));
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    // times the keys' scales; the largest of the row
    float mx = -INFINITY;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 ks = *reinterpret_cast<const f32x4*>(rec + R::KS + 4 * (32 * x + 8 * k + 4 * h));
#pragma unroll
        for (int c = 0; c < 4; ++c) s[x][4 * k + c] *= ks[c];
      }
    if (!whole) {
      const uint64_t mine_bits = bits >> (4 * h);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int n = 32 * x + 8 * (k >> 2) + (k & 3);
          const bool see = (((mine_bits >> n) & 1) != 0) & range.sees(j0 + n + 4 * h);
          s[x][k] = see ? s[x][k] : -INFINITY;
        }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int k = 0; k < 16; k += 2) mx = max3(mx, s[x][k], s[x][k + 1]);
    // new references only where these tokens might pass the present ones (-infinity stays so)
    mx *= q_scale;
    if (__any(sum.passed(mx, *reinterpret_cast<const float*>(rec + R::TOP)))) {
      float both = -INFINITY;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f32x4 vs = *reinterpret_cast<const f32x4*>(rec + R::VS + 4 * (32 * x + 8 * k + 4 * h));
#pragma unroll
          for (int c = 0; c < 4; ++c)
            both = fmaxf(both, __builtin_fmaf(s[x][4 * k + c], q_scale, __builtin_amdgcn_logf(finite_size(vs[c]))));
        }
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      both = fmaxf(both, __shfl_xor(both, 32, 64));
      const float f = sum.raise(mx, both);
      if (__any(f != 1.0f)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= f;
      }
    }

    uint32_t pop[2][16];   // pairs of weights, two terms: operand k holds words 4 k ..
    float part[2] = {};
    auto weights = [&](auto plain) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f32x4 vs = *reinterpret_cast<const f32x4*>(rec + R::VS + 4 * (32 * x + 8 * k + 4 * h));
#pragma unroll
          for (int c = 0; c < 4; c += 2) {
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float v = s[x][4 * k + c + e], d = __builtin_fmaf(v, q_scale, -sum.ref);
              if constexpr (decltype(plain)::value) {
                const float p = __builtin_amdgcn_exp2f(d);
                part[e] += p;
                w[e] = p * vs[c + e];
              } else {
                part[e] += sum.term(d, __builtin_fmaf(v, q_scale, -sum.m), vs[c + e], w[e]);
                w[e] = v == -INFINITY ? 0.0f : w[e];
              }
            }
            const int at = 8 * x + 2 * k + (c >> 1);
            two_terms(w[0], w[1], pop[0][at], pop[1][at]);
          }
        }
    };
    // tokens that are not seen have weight 0 also where their scale is not a number
    if (!sum.wide && (whole || *reinterpret_cast<const uint32_t*>(rec + R::FINITE))) {
      weights(std::true_type{});
    } else {
      weights(std::false_type{});
    }
    sum.add(part[0] + part[1]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const h8 v = vop[d & 1][k];
        if (d + 2 < DT)
          vop[d & 1][k] = *reinterpret_cast<const h8*>(rec + R::V + ((((d + 2) * 4 + k) * 64 + lane) << 4));
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const u32x4 w = {pop[y][4 * k], pop[y][4 * k + 1], pop[y][4 * k + 2], pop[y][4 * k + 3]};
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, __builtin_bit_cast(h8, w), o[d], 0, 0, 0);
        }
      }
    }
  }

  const float l = sum.l + __shfl_xor(sum.l, 32, 64);
  if (!there) return;
  // o holds the sums over V relative to 2^ref
  const float f = half_power(sum.ref - sum.m);
  const int64_t token = sq.first + i;
  if (a.chunks == 1) {
    const float inv = f * a.v_scale * inverse_sum(l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        store_out(a.out, a.dtype, token * a.out_token + hq * a.out_head + 32 * d + 8 * k + 4 * h,
                  f32x4{o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]} * f * inv);
    if (a.lse && h == 0)
      a.lse[token * a.q_heads + hq] = log_sum(sum.m, l);
  } else {
    float* p = partial(a, b, head, rb, 32 * wave + t, chunk, DIM);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<f32x4*>(p + 4 + 32 * d + 8 * k + 4 * h) =
            f32x4{o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]} * f * (f * a.v_scale);
    if (h == 0) {
      p[0] = sum.m;
      p[1] = l;
    }
  }
}

template <int DIM>
hipError_t launch(const AttendArgs& a, int decoder, hipStream_t st) {
  const dim3 each((unsigned)(a.groups * a.heads * a.seqs));
  if (decoder) {
    hipLaunchKernelGGL((unpack_kernel<DIM, true>), each, dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL((unpack_kernel<DIM, false>), each, dim3(256), 0, st, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(a.chunks * a.blocks * a.heads * a.seqs));
  constexpr int bytes = 2 * Record<DIM>::BYTES;
  if (a.dtype == NQ_F32) {
    hipLaunchKernelGGL((prompt_kernel<DIM, 2>), grid, dim3(64 * kWaves), bytes, st, a);
  } else {
    hipLaunchKernelGGL((prompt_kernel<DIM, 1>), grid, dim3(64 * kWaves), bytes, st, a);
  }
  e = hipGetLastError();
  return e == hipSuccess && a.chunks > 1 ? launch_join<DIM, kRows, 6, 1>(a, st) : e;
}

template <int DIM>
hipError_t attributes() {
  for (const void* f : {(const void*)prompt_kernel<DIM, 1>, (const void*)prompt_kernel<DIM, 2>}) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             2 * Record<DIM>::BYTES);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t prompt_set_attributes() {
  hipError_t e = attributes<64>();
  if (e == hipSuccess) e = attributes<128>();
  if (e == hipSuccess) e = attributes<256>();
  return e;
}

hipError_t launch_prompt(const AttendArgs& a, int dim, int decoder, hipStream_t st) {
  switch (dim) {
    case 64: return launch<64>(a, decoder, st);
    case 128: return launch<128>(a, decoder, st);
    default: return launch<256>(a, decoder, st);
  }
}

}  // namespace nq
