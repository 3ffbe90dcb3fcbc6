// Selection of cache blocks by the bounds of their keys (gfx950).
//
// For a group of query rows (tokens x query heads of one KV head) the score of a block with smallest / largest keys lo, hi is
//     max over rows r of  sum_d q_rd (q_rd > 0 ? hi_d : lo_d)  =  max_r ( min(q_r, 0) . lo + max(q_r, 0) . hi ),
// the largest value that any q_r . k of the block could have.  The blocks with the largest scores are taken, ties to the lower
// index; the first and the last few are taken whatever they score.
//
// The sums are products of inner length 2 D and run on the matrix cores with fp32 accumulators.  Their rounding must not
// decide between two blocks, so a first pass only sorts out what is beyond doubt: with e a bound of every rounded score's
// error and t the rounded score of rank n, a block above t + 2 e is certainly taken and one below t - 2 e certainly not
// (the exact score of rank n is within e of t).  What lies between is evaluated in fp64, where products of bf16 numbers are
// exact and their sums of 2 D terms as good as exact, and ranked by that.
#include "attn_common.hpp"

namespace la {
namespace {

// Error of a rounded score relative to sum_d |q_d| max(|lo_d|, |hi_d|): at most 2 D <= 512 additions, each off by at most a
// unit in the last place of a partial sum (2^-23, whichever way the matrix core rounds).
template <int D>
constexpr float kScoreError = 2.0f * D / (1 << 23);

__device__ __forceinline__ uint32_t order_key(float x) {  // larger numbers have larger keys
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t order_key64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return u >> 63 ? ~u : u | (1ull << 63);
}

__device__ __forceinline__ int prefix_blocks(const SelectParams &p, int b) {
  const int P = (int)min((int64_t)max(p.prefix_lens[b], 0), (int64_t)p.max_blocks << p.block_shift);
  return min((P + (1 << p.block_shift) - 1) >> p.block_shift, p.n_max);
}

// The negative and the other elements of eight bf16 numbers.
__device__ __forceinline__ void split_signs(const u32x4 q, u32x4 &neg, u32x4 &pos) {
  typedef __attribute__((ext_vector_type(2))) short i16x2;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = q[i];  // (a bit cast of a vector's element would take the vector's first one)
    const uint32_t mask = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, w) >> 15);
    neg[i] = w & mask, pos[i] = w & ~mask;
  }
}

// A wavefront scores 32 blocks for one group: their bounds stay in registers as matrix operands while the group's rows pass,
// 32 at a time; the largest of a block's row sums is then a maximum over registers.
template <int D>
__global__ __launch_bounds__(256) void block_score_kernel(const SelectParams p) {
  constexpr int T = D / 16;
  const int lane = threadIdx.x & 63, ln = lane & 31, h = lane >> 5;
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  uint32_t id = blockIdx.y + blockIdx.z * 65535u;
  if (id >= (uint32_t)(p.B * p.gamma * p.n_groups * p.Hkv)) return;
  const size_t unit = id;
  const int hk = (int)(id % (uint32_t)p.Hkv);
  id /= (uint32_t)p.Hkv;
  const int per_req = p.gamma * p.n_groups;
  const int b = (int)(id / (uint32_t)per_req), group = (int)(id % (uint32_t)per_req);
  const int n = prefix_blocks(p, b);
  if (n <= p.max_sel || tile * 32 >= n) return;  // all blocks are taken / no such blocks
  const int lb = min(tile * 32 + ln, n - 1);
  const int blk = p.block_tables ? p.block_tables[(size_t)b * p.max_blocks + lb] : b * p.max_blocks + lb;
  const uint8_t *src = (const uint8_t *)p.k_bounds + ((size_t)blk * p.Hkv + hk) * 4 * D + h * 16;
  u32x4 lo[T], hi[T];
#pragma unroll
  for (int t = 0; t < T; ++t) lo[t] = *(const u32x4 *)(src + t * 32), hi[t] = *(const u32x4 *)(src + 2 * D + t * 32);

  const int g = group / p.n_groups, t0 = (group - g * p.n_groups) * p.group_len;
  const int n_rows = min(p.group_len, p.L - t0) * p.G;
  const size_t tok0 = ((size_t)b * p.gamma + g) * p.L + t0;
  float best = -INFINITY;
  for (int r0 = 0; r0 < n_rows; r0 += 32) {
    const int r = min(r0 + ln, n_rows - 1);  // surplus rows repeat the last one
    const uint8_t *qs = (const uint8_t *)p.q + ((tok0 + r / p.G) * p.Hq + hk * p.G + r % p.G) * D * 2 + h * 16;
    f32x16 s;
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      u32x4 neg, pos;
      split_signs(*(const u32x4 *)(qs + t * 32), neg, pos);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, neg), __builtin_bit_cast(bf16x8, lo[t]), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, pos), __builtin_bit_cast(bf16x8, hi[t]), s, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) best = fmaxf(best, s[j]);
  }
  best = xhalf_max(best);
  if (h == 0 && tile * 32 + ln < n) p.score[unit * p.n_max + tile * 32 + ln] = best;
  if (group == 0) {  // the largest magnitude among the tile's bounds, once per request and head
    uint32_t top = 0;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top = max(top, max(lo[t][i] << 16 & 0x7fffffffu, lo[t][i] & 0x7fff0000u));
        top = max(top, max(hi[t][i] << 16 & 0x7fffffffu, hi[t][i] & 0x7fff0000u));
      }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
    if (lane == 0) p.top[((size_t)b * p.Hkv + hk) * p.n_tiles + tile] = __builtin_bit_cast(float, top);
  }
}

// Rank n (1 = the largest) among the keys of items 0 .. count - 1 that `key_of` gives (0: not an item): the key, and how
// many items above it there are.  Eight bits at a time; every thread of the workgroup calls it.
template <typename Key, typename F>
__device__ Key key_of_rank(int count, int n, F key_of, int *above, uint32_t (&hist)[256], uint32_t (&found)[2]) {
  Key prefix = 0;
  int left = n;
  for (int shift = (int)sizeof(Key) * 8 - 8; shift >= 0; shift -= 8) {
    hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += 256) {
      const Key k = key_of(i);
      if (k != 0 && (shift + 8 >= (int)sizeof(Key) * 8 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
        atomicAdd(&hist[(uint32_t)(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t run = 0;
      int d = 255;
      for (; d > 0 && run + hist[d] < (uint32_t)left; --d) run += hist[d];
      found[0] = (uint32_t)d, found[1] = run;
    }
    __syncthreads();
    prefix |= (Key)found[0] << shift;
    left -= (int)found[1];
    __syncthreads();
  }
  *above = n - left;
  return prefix;
}

constexpr int kListed = 1024;  // blocks in doubt that are evaluated at a time

// One workgroup picks the blocks of one group and KV head from their scores.
template <int D>
__global__ __launch_bounds__(256) void block_pick_kernel(const SelectParams p) {
  __shared__ uint32_t hist[256], found[2];
  __shared__ float red[4];
  __shared__ int list[kListed], n_list, wave_count[4][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t id = blockIdx.x;
  const size_t unit = id;
  const int hk = (int)(id % (uint32_t)p.Hkv);
  id /= (uint32_t)p.Hkv;
  const int per_req = p.gamma * p.n_groups;
  const int b = (int)(id / (uint32_t)per_req), group = (int)(id % (uint32_t)per_req);
  const int n = prefix_blocks(p, b);
  int32_t *out = p.blocks + unit * p.max_sel;
  if (n <= p.max_sel) {
    for (int i = tid; i < p.max_sel; i += 256) out[i] = i < n ? i : -1;
    if (tid == 0) p.count[unit] = n;
    return;
  }
  const int c0 = p.keep_first, c1 = n - p.keep_last;           // candidates
  const int want = p.max_sel - p.keep_first - p.keep_last;     // fewer than there are
  const float *score = p.score + unit * p.n_max;
  double *exact = p.exact + unit * p.n_max;

  // the largest sum of magnitudes of a row, the largest magnitude of a bound: the error of the scores
  const int g = group / p.n_groups, t0 = (group - g * p.n_groups) * p.group_len;
  const int n_rows = min(p.group_len, p.L - t0) * p.G;
  const size_t tok0 = ((size_t)b * p.gamma + g) * p.L + t0;
  auto row_of = [&](int r) __attribute__((always_inline)) {
    return (const uint8_t *)p.q + ((tok0 + r / p.G) * p.Hq + hk * p.G + r % p.G) * D * 2;
  };
  float size_q = 0.f, size_k = 0.f;
  constexpr int kPer = D / 8;  // lanes that share a row
  for (int i0 = 0; i0 < n_rows * kPer; i0 += 256) {
    const int i = i0 + tid;
    float a = 0.f;
    if (i < n_rows * kPer) {
      const u32x4 x = *(const u32x4 *)(row_of(i / kPer) + (i % kPer) * 16);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        a += __builtin_bit_cast(float, x[w] << 16 & 0x7fffffffu) + __builtin_bit_cast(float, x[w] & 0x7fff0000u);
    }
#pragma unroll
    for (int off = 1; off < kPer; off <<= 1) a += __shfl_xor(a, off);
    size_q = fmaxf(size_q, a);
  }
  for (int i = tid; i < (n + 31) / 32; i += 256) size_k = fmaxf(size_k, p.top[((size_t)b * p.Hkv + hk) * p.n_tiles + i]);
  auto all_max = [&](float v) __attribute__((always_inline)) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v = fmaxf(v, __shfl_xor(v, off));
    __syncthreads();
    if (lane == 0) red[wave] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  };
  size_q = all_max(size_q), size_k = all_max(size_k);
  const float err = kScoreError<D> * 1.01f * size_q * size_k + 1e-30f;

  float sure = INFINITY, out_of = INFINITY;  // above: certainly taken; below: certainly not
  int above = 0, need = 0, n_doubt = 0;
  if (want > 0) {
    int rank_above;
    const uint32_t kt = key_of_rank<uint32_t>(
        c1 - c0, want, [&](int i) { return order_key(score[c0 + i]); }, &rank_above, hist, found);
    const float t = key_value(kt);
    sure = t + 2.f * err, out_of = t - 2.f * err;
    int mine_sure = 0, mine_doubt = 0;
    for (int i = c0 + tid; i < c1; i += 256) {
      const float s = score[i];
      mine_sure += s > sure ? 1 : 0, mine_doubt += s >= out_of && !(s > sure) ? 1 : 0;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) mine_sure += __shfl_xor(mine_sure, off), mine_doubt += __shfl_xor(mine_doubt, off);
    if (lane == 0) wave_count[wave][0] = mine_sure, wave_count[wave][1] = mine_doubt;
    __syncthreads();
    for (int w = 0; w < 4; ++w) above += wave_count[w][0], n_doubt += wave_count[w][1];
    need = want - above;
    __syncthreads();
  }
  auto in_doubt = [&](float s) __attribute__((always_inline)) { return s >= out_of && !(s > sure); };

  uint64_t exact_t = 0;
  int ties = n_doubt;  // blocks at the threshold that are taken, the lowest indices first
  if (n_doubt > need) {
    // exact scores of the blocks in doubt
    auto evaluate = [&](int count) __attribute__((always_inline)) {
      const int part = lane & 7, r8 = lane >> 3;
      for (int k = wave; k < count; k += 4) {
        const int lb = list[k];
        const int blk = p.block_tables ? p.block_tables[(size_t)b * p.max_blocks + lb] : b * p.max_blocks + lb;
        const uint8_t *bs = (const uint8_t *)p.k_bounds + ((size_t)blk * p.Hkv + hk) * 4 * D;
        double best = -INFINITY;
        for (int r0 = 0; r0 < n_rows; r0 += 8) {
          const uint8_t *qs = row_of(min(r0 + r8, n_rows - 1));
          double sum = 0.0;
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const int at = (c * 8 + part) * 16;
            const u32x4 q = *(const u32x4 *)(qs + at), lo = *(const u32x4 *)(bs + at), hi = *(const u32x4 *)(bs + 2 * D + at);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t a = (q[w] << 16) >> 31 ? lo[w] << 16 : hi[w] << 16;
              const uint32_t z = q[w] >> 31 ? lo[w] & 0xffff0000u : hi[w] & 0xffff0000u;
              sum += (double)__builtin_bit_cast(float, q[w] << 16) * (double)__builtin_bit_cast(float, a);
              sum += (double)__builtin_bit_cast(float, q[w] & 0xffff0000u) * (double)__builtin_bit_cast(float, z);
            }
          }
          sum += __shfl_xor(sum, 1), sum += __shfl_xor(sum, 2), sum += __shfl_xor(sum, 4);
          best = fmax(best, sum);
        }
        best = fmax(best, __shfl_xor(best, 8)), best = fmax(best, __shfl_xor(best, 16)), best = fmax(best, __shfl_xor(best, 32));
        if (lane == 0) exact[lb] = best;
      }
    };
    if (tid == 0) n_list = 0;
    __syncthreads();
    for (int i0 = c0; i0 < c1; i0 += 256) {
      const int i = i0 + tid;
      if (i < c1 && in_doubt(score[i])) list[atomicAdd(&n_list, 1)] = i;
      __syncthreads();
      const int count = n_list;
      if (count > kListed - 256 || i0 + 256 >= c1) {
        evaluate(count);
        __syncthreads();
        if (tid == 0) n_list = 0;
      }
      __syncthreads();
    }
    int exact_above;
    exact_t = key_of_rank<uint64_t>(
        c1 - c0, need, [&](int i) { return in_doubt(score[c0 + i]) ? order_key64(exact[c0 + i]) : 0ull; }, &exact_above, hist,
        found);
    ties = need - exact_above;
  }

  // the list, in ascending order
  int at = 0, tied = 0;
  for (int i0 = 0; i0 < n; i0 += 256) {
    const int i = i0 + tid;
    bool take = i < n && (i < c0 || i >= c1), tie = false;
    if (i >= c0 && i < c1 && want > 0) {
      const float s = score[i];
      if (s > sure) {
        take = true;
      } else if (in_doubt(s)) {
        if (n_doubt > need) {
          const uint64_t k = order_key64(exact[i]);
          take = k > exact_t, tie = k == exact_t;
        } else {
          take = true;
        }
      }
    }
    const uint64_t tie_mask = __builtin_amdgcn_ballot_w64(tie), below = (1ull << lane) - 1;
    if (lane == 0) wave_count[wave][1] = __popcll(tie_mask);
    __syncthreads();
    int rank = tied + __popcll(tie_mask & below);
    for (int w = 0; w < 4; ++w) rank += w < wave ? wave_count[w][1] : 0, tied += wave_count[w][1];
    take |= tie && rank < ties;
    const uint64_t mask = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) wave_count[wave][0] = __popcll(mask);
    __syncthreads();
    int place = at + __popcll(mask & below);
    for (int w = 0; w < 4; ++w) place += w < wave ? wave_count[w][0] : 0, at += wave_count[w][0];
    if (take && place < p.max_sel) out[place] = i;
    __syncthreads();
  }
  for (int i = at + tid; i < p.max_sel; i += 256) out[i] = -1;
  if (tid == 0) p.count[unit] = min(at, p.max_sel);
}

template <int D>
hipError_t launch(const SelectParams &p, hipStream_t stream) {
  const int64_t units = (int64_t)p.B * p.gamma * p.n_groups * p.Hkv;
  if (p.n_max > p.max_sel) {
    ProfileScope scope(SLOT_BLOCK_SCORE, stream);
    const dim3 grid((unsigned)((p.n_tiles + 3) / 4), (unsigned)(units < 65535 ? units : 65535), (unsigned)((units + 65534) / 65535));
    hipLaunchKernelGGL((block_score_kernel<D>), grid, dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfileScope scope(SLOT_BLOCK_PICK, stream);
  hipLaunchKernelGGL((block_pick_kernel<D>), dim3((unsigned)units), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_select(const SelectParams &p, hipStream_t stream) {
  switch (p.D) {
    case 64: return launch<64>(p, stream);
    case 128: return launch<128>(p, stream);
    case 256: return launch<256>(p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace la
