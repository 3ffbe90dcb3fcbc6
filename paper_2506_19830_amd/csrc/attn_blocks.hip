// Verification attention over selected blocks of a block cache (gfx950).
//
// Every group of query tokens and KV head has a list of blocks of the prefix; its rows (tokens x query heads of the KV head)
// attend to the keys of these blocks and to the branch's own tokens up to their own:
//     out = softmax(scale q.k) v   over both,   one pass with the running maximum and sum.
//
// A wavefront owns 32 (or 64) rows and walks over tiles of 32 keys on its own; the four wavefronts of a workgroup, and the
// workgroups that share a unit, have disjoint tiles and are folded at the end.  The products are transposed:
//     S^T (32 keys x 32 rows) = K Q^T,   O^T (D x 32 rows) += V^T P^T
// so that a lane holds scores of one row only, and P^T leaves the accumulators of the first product in the order in which
// the second one wants its operand (the keys of a tile are permuted alike on both sides).
//   K goes from memory into matrix operands through registers alone: the lane of key n and half h holds the elements
//     d = h D/2 .. of its row, 16 bytes per load, and the inner index of the product is permuted to match (Q likewise).
//   V is widened to bf16 on its way into LDS (8 KB per wavefront at D = 128) and read back transposed by 16-bit reads.
//   Quantised rows are widened exactly, with their exponents applied by the conversion.
// Probabilities are rounded to bf16 for the second product (relative 2^-9 each, of the size of the output's own rounding);
// scores, maxima, sums and accumulators are fp32.
#include "attn_common.hpp"

namespace la {
namespace {

constexpr int kWaves = 4;
constexpr int kMaxSlots = 2048;  // blocks whose place a workgroup holds in LDS

// The half row of one key, as stored.
template <int FMT, int D>
struct Raw {
  static constexpr int kWords = FMT == FMT_BF16 ? D / 4 : FMT == FMT_MX8 ? D / 8 : D / 16;
  uint32_t w[kWords];
  uint32_t e;  // exponents of the D / 64 groups, a byte each
};

template <int FMT, int D>
__device__ __forceinline__ void load_half(Raw<FMT, D> &r, const void *base, const uint8_t *exps, size_t row, int h) {
  const uint8_t *src = (const uint8_t *)base + (row * 2 + h) * (Raw<FMT, D>::kWords * 4);
#pragma unroll
  for (int i = 0; i < Raw<FMT, D>::kWords; i += 4) {
    const u32x4 x = *(const u32x4 *)(src + i * 4);
    r.w[i] = x[0], r.w[i + 1] = x[1], r.w[i + 2] = x[2], r.w[i + 3] = x[3];
  }
  if constexpr (FMT != FMT_BF16) {
    const uint8_t *pe = exps + (row * 2 + h) * (D / 64);
    if constexpr (D == 64)
      r.e = *pe;
    else if constexpr (D == 128)
      r.e = *(const uint16_t *)pe;
    else
      r.e = *(const uint32_t *)pe;
  }
}

// Elements 8 t .. 8 t + 7 of the half row as four bf16 pairs.
template <int FMT, int D>
__device__ __forceinline__ u32x4 widen(const Raw<FMT, D> &r, int t) {
  u32x4 x;
  if constexpr (FMT == FMT_BF16) {
    x = u32x4{r.w[4 * t], r.w[4 * t + 1], r.w[4 * t + 2], r.w[4 * t + 3]};
  } else {
    const float s = __builtin_bit_cast(float, ((r.e >> (8 * (t / 4))) & 0xffu) << 23);
    if constexpr (FMT == FMT_MX8) {
      x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.w[2 * t], s, false));
      x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.w[2 * t], s, true));
      x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.w[2 * t + 1], s, false));
      x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.w[2 * t + 1], s, true));
    } else {
      x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[t], s, 0));
      x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[t], s, 1));
      x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[t], s, 2));
      x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[t], s, 3));
    }
  }
  return x;
}

// The 16-byte pieces of a V row lie permuted in LDS, piece c of key k at c ^ swizzle(k): the 16 keys that one store
// instruction writes at a time, and the four keys x 64 bytes that one transposing read gathers, then fall into different
// banks.
template <int D>
__device__ __forceinline__ int swizzle(int key) {
  return D == 64 ? (((key >> 1) & 1) << 2) | ((key >> 2) & 3) : ((key & 3) << 2) | ((key >> 2) & 3);
}

typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

template <int D, int RB>
struct Rows {
  bf16x8 q[RB][D / 16];
  f32x16 o[RB][D / 32];
  float m[RB], l[RB];          // running maximum (log2 units) and this lane's share of the sum
  int tok[RB], start[RB];      // token of the row inside the request, first token of its branch
};

enum TileMask { TILE_FULL = 0, TILE_TAIL, TILE_OWN };

// Scores of one tile from the K half rows, then probabilities, then the product with the V tile in LDS.
// first: index of the tile's first key; limit: keys from there on do not exist (TILE_TAIL).
template <int D, int RB, int MASK>
__device__ __forceinline__ void attend(Rows<D, RB> &st, f32x16 (&s)[RB], const uint8_t *vt, float scale_log2, int first,
                                       int limit, int lane) {
  const int h = lane >> 5;
  float alpha[RB];
  bool raise = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int key = first + (j >> 2) * 8 + h * 4 + (j & 3);
      s[rb][j] *= scale_log2;
      if constexpr (MASK == TILE_TAIL) {
        if (key >= limit) s[rb][j] = -INFINITY;
      } else if constexpr (MASK == TILE_OWN) {
        if (key > st.tok[rb] || key < st.start[rb]) s[rb][j] = -INFINITY;
      }
      top = fmaxf(top, s[rb][j]);
    }
    top = xhalf_max(top);
    // the maximum is raised only when a tile exceeds it by kRaise: until then probabilities may reach 2^kRaise
    const bool up = top > st.m[rb] + kRaise;
    const float m = up ? top : st.m[rb];
    alpha[rb] = up ? __builtin_amdgcn_exp2f(st.m[rb] - m) : 1.0f;
    st.m[rb] = m;
    raise |= up;
  }
  if (__builtin_amdgcn_ballot_w64(raise)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      st.l[rb] *= alpha[rb];
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) st.o[rb][db][j] *= alpha[rb];
    }
  }
  bf16x8 pf[RB][2];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float base = st.m[rb] == -INFINITY ? 0.f : st.m[rb];  // no key seen yet: every score is -inf
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(s[rb][8 * c + 2 * i] - base);
        const float p1 = __builtin_amdgcn_exp2f(s[rb][8 * c + 2 * i + 1] - base);
        sum += p0 + p1;
        w[i] = pack_bf16(p0, p1);
      }
      pf[rb][c] = __builtin_bit_cast(bf16x8, w);
    }
    st.l[rb] += sum;
  }
  // V^T operands: lane (d, h) takes keys 16 c + 4 h + 0..3 and + 8, the order of the probabilities above
  const int i = lane & 15, sub = (lane >> 4) & 1;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = 16 * c + 8 * e + 4 * h + (i >> 2);
        const int piece = (4 * db + 2 * sub + ((i & 3) >> 1)) ^ swizzle<D>(key);
        const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vt + key * D * 2 + piece * 16 + (i & 1) * 8));
        const u32x2 y = __builtin_bit_cast(u32x2, x);
        w[2 * e] = y[0], w[2 * e + 1] = y[1];
      }
      const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        st.o[rb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[rb][c], st.o[rb][db], 0, 0, 0);
    }
}

template <int FMT, int D, int RB>
__device__ __forceinline__ void scores(f32x16 (&s)[RB], const Raw<FMT, D> &k, const Rows<D, RB> &st) {
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int j = 0; j < 16; ++j) s[rb][j] = 0.f;
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    const bf16x8 kf = __builtin_bit_cast(bf16x8, widen<FMT, D>(k, t));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, st.q[rb][t], s[rb], 0, 0, 0);
  }
}

template <int FMT, int D>
__device__ __forceinline__ void stage_v(uint8_t *vt, const Raw<FMT, D> &v, int key, int h) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    const int piece = (h * (D / 16) + t) ^ swizzle<D>(key);
    *(u32x4 *)(vt + key * D * 2 + piece * 16) = widen<FMT, D>(v, t);
  }
}

// LDS written by some lanes is read by others of the same wavefront: the compiler must not move one across the other (the
// hardware keeps a wavefront's LDS operations in order).
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int FMT, int D, int RB>
__global__ __launch_bounds__(256, RB == 1 && D <= 128 ? 2 : 1) void attn_blocks_kernel(const SparseParams p) {
  constexpr int kTileBytes = 32 * D * 2;                 // V tile of a wavefront
  constexpr int kFoldBytes = 2 * RB * (D / 32) * 16 * 64 * 4;  // accumulators of two wavefronts
  constexpr int kBytes = kWaves * kTileBytes > kFoldBytes ? kWaves * kTileBytes : kFoldBytes;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kBytes];
  __shared__ int32_t place[kMaxSlots];
  __shared__ float fold_ml[kWaves][RB * 32][2];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ln = lane & 31, h = lane >> 5;
  // KV heads vary fastest: with eight of them each XCD keeps to one head's keys
  uint32_t id = blockIdx.x;
  const int hk = (int)(id % (uint32_t)p.Hkv);
  id /= (uint32_t)p.Hkv;
  const int split = (int)(id % (uint32_t)p.n_split);
  id /= (uint32_t)p.n_split;
  const int row_tile = (int)(id % (uint32_t)p.n_row_tiles);
  id /= (uint32_t)p.n_row_tiles;
  const int group = (int)(id % (uint32_t)p.n_groups), b = (int)(id / (uint32_t)p.n_groups);

  // rows of the unit
  int tok0 = 0, n_tok = p.gamma * p.L;
  if (p.sel) {
    const int per_branch = p.n_groups / p.gamma, g = group / per_branch, t0 = (group - g * per_branch) * p.group_len;
    tok0 = g * p.L + t0;
    n_tok = min(p.group_len, p.L - t0);
  }
  const int n_group_rows = n_tok * p.G, r0 = row_tile * (RB * 32);
  if (r0 >= n_group_rows) return;
  const int r_last = min(r0 + RB * 32, n_group_rows) - 1;
  const int own0 = (tok0 + r0 / p.G) / p.L * p.L, own_end = tok0 + r_last / p.G + 1;  // own tokens any row sees

  // keys of the prefix
  const int bs = 1 << p.block_shift;
  const int P = (int)min((int64_t)max(p.prefix_lens[b], 0), (int64_t)p.max_blocks << p.block_shift);
  const int n_blocks = (P + bs - 1) >> p.block_shift;
  const size_t unit = ((size_t)b * p.n_groups + group) * p.Hkv + hk;
  const int32_t *list = p.sel ? p.sel + unit * p.max_sel : nullptr;
  int n_keys = P;
  if (p.sel) {
    const int n = min(max(p.sel_count[unit], 0), min(p.max_sel, n_blocks));
    n_keys = 0;
    if (n > 0) {
      const int last = min(max(list[n - 1], 0), n_blocks - 1);
      n_keys = ((n - 1) << p.block_shift) + min(bs, P - (last << p.block_shift));
    }
  }
  const int n_tiles = (n_keys + 31) >> 5, n_own_tiles = (own_end - own0 + 31) >> 5;
  const int64_t total = (int64_t)n_tiles + n_own_tiles, slots = (int64_t)p.n_split * kWaves;
  const int s0 = split * kWaves;
  const int wg_begin = (int)(s0 * total / slots), wg_end = (int)((s0 + kWaves) * total / slots);
  const int begin = (int)((s0 + wave) * total / slots), end = (int)((s0 + wave + 1) * total / slots);

  // where the blocks of the workgroup's tiles lie
  const int slot0 = (wg_begin * 32) >> p.block_shift;
  if (wg_begin < min(wg_end, n_tiles)) {
    const int slot_end = ((min(wg_end * 32, n_keys) - 1) >> p.block_shift) + 1;
    for (int i = threadIdx.x; i < slot_end - slot0; i += 256) {
      const int lb = list ? min(max(list[slot0 + i], 0), n_blocks - 1) : slot0 + i;
      const int blk = p.block_tables ? p.block_tables[(size_t)b * p.max_blocks + lb] : b * p.max_blocks + lb;
      place[i] = blk;
    }
  }

  Rows<D, RB> st;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = min(r0 + rb * 32 + ln, n_group_rows - 1);
    const int tok = tok0 + r / p.G, head = hk * p.G + r % p.G;
    const uint8_t *src = (const uint8_t *)p.q + (((size_t)b * p.gamma * p.L + tok) * p.Hq + head) * D * 2 + h * D;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) st.q[rb][t] = *(const bf16x8 *)(src + t * 16);
    st.tok[rb] = tok, st.start[rb] = tok / p.L * p.L;
    st.m[rb] = -INFINITY, st.l[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) st.o[rb][db][j] = 0.f;
  }
  __syncthreads();

  uint8_t *vt = lds + wave * kTileBytes;
  // the prefix: the rows of the next tile are requested before the present one is used
  const int pre_end = min(end, n_tiles);
  if (begin < pre_end) {
    auto row_of = [&](int tile) __attribute__((always_inline)) {
      const int key = min(tile * 32 + ln, n_keys - 1);
      const int blk = place[(key >> p.block_shift) - slot0];
      return ((((size_t)blk * p.Hkv + hk) << p.block_shift) + (key & (bs - 1)));
    };
    Raw<FMT, D> k, v;
    size_t row = row_of(begin);
    load_half(k, p.k_cache, p.k_exp, row, h);
    load_half(v, p.v_cache, p.v_exp, row, h);
    for (int tile = begin; tile < pre_end; ++tile) {
      const size_t next = row_of(min(tile + 1, pre_end - 1));
      stage_v(vt, v, ln, h);
      load_half(v, p.v_cache, p.v_exp, next, h);
      f32x16 s[RB];
      scores(s, k, st);
      load_half(k, p.k_cache, p.k_exp, next, h);
      wave_order();
      if ((tile + 1) * 32 <= n_keys)
        attend<D, RB, TILE_FULL>(st, s, vt, p.scale_log2, tile * 32, n_keys, lane);
      else
        attend<D, RB, TILE_TAIL>(st, s, vt, p.scale_log2, tile * 32, n_keys, lane);
      wave_order();
    }
  }
  // the branch's own tokens
  for (int tile = max(begin, n_tiles); tile < end; ++tile) {
    const int first = own0 + (tile - n_tiles) * 32;
    const size_t row = ((size_t)b * p.gamma * p.L + min(first + ln, own_end - 1)) * p.Hkv + hk;
    Raw<FMT_BF16, D> k, v;
    load_half(k, p.k_branch, nullptr, row, h);
    load_half(v, p.v_branch, nullptr, row, h);
    stage_v(vt, v, ln, h);
    f32x16 s[RB];
    scores(s, k, st);
    wave_order();
    attend<D, RB, TILE_OWN>(st, s, vt, p.scale_log2, first, own_end, lane);
    wave_order();
  }

  // fold the four wavefronts: common maximum, then the accumulators pairwise through LDS
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    st.l[rb] = xhalf_sum(st.l[rb]);
    if (h == 0) fold_ml[wave][rb * 32 + ln][0] = st.m[rb], fold_ml[wave][rb * 32 + ln][1] = st.l[rb];
  }
  __syncthreads();  // (also: every wavefront is done with its V tile)
  float m_all[RB], l_all[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_all[rb] = -INFINITY, l_all[rb] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m_all[rb] = fmaxf(m_all[rb], fold_ml[w][rb * 32 + ln][0]);
    const float base = m_all[rb] == -INFINITY ? 0.f : m_all[rb];
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      l_all[rb] += fold_ml[w][rb * 32 + ln][1] * __builtin_amdgcn_exp2f(fold_ml[w][rb * 32 + ln][0] - base);
    const float f = __builtin_amdgcn_exp2f(st.m[rb] - base);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) st.o[rb][db][j] *= f;
  }
  constexpr int kOne = RB * (D / 32) * 16 * 64;  // floats of one wavefront's accumulators
  float *buf = (float *)lds;
  auto put = [&](float *dst) __attribute__((always_inline)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) dst[((rb * (D / 32) + db) * 16 + j) * 64 + lane] = st.o[rb][db][j];
  };
  auto add = [&](const float *src) __attribute__((always_inline)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) st.o[rb][db][j] += src[((rb * (D / 32) + db) * 16 + j) * 64 + lane];
  };
  if (wave & 1) put(buf + (wave >> 1) * kOne);
  __syncthreads();
  if (!(wave & 1)) add(buf + (wave >> 1) * kOne);
  __syncthreads();
  if (wave == 2) put(buf);
  __syncthreads();
  if (wave != 0) return;
  add(buf);

  const size_t all_rows = (size_t)p.B * p.n_rows;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = r0 + rb * 32 + ln;
    if (r >= n_group_rows) continue;
    const size_t grow = (size_t)b * p.n_rows + (size_t)(tok0 + r / p.G) * p.Hq + hk * p.G + r % p.G;
    if (p.part_o) {
      const size_t prow = split * all_rows + grow;
      if (h == 0) *(f32x2 *)(p.part_ml + prow * 2) = f32x2{m_all[rb], l_all[rb]};
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(f32x4 *)(p.part_o + prow * D + db * 32 + q * 8 + h * 4) =
              f32x4{st.o[rb][db][4 * q], st.o[rb][db][4 * q + 1], st.o[rb][db][4 * q + 2], st.o[rb][db][4 * q + 3]};
      continue;
    }
    const float inv = 1.0f / l_all[rb];
    if (p.lse && h == 0) p.lse[grow] = 0.69314718055994530942f * (m_all[rb] + __builtin_log2f(l_all[rb]));
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = f32x4{st.o[rb][db][4 * q], st.o[rb][db][4 * q + 1], st.o[rb][db][4 * q + 2], st.o[rb][db][4 * q + 3]} * inv;
        const size_t at = grow * D + db * 32 + q * 8 + h * 4;
        if (p.out_f32)
          *(f32x4 *)((float *)p.out + at) = x;
        else
          *(u32x2 *)((uint8_t *)p.out + at * 2) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
      }
  }
}

template <int FMT, int D>
hipError_t launch(const SparseParams &p, hipStream_t stream) {
  const int64_t units = (int64_t)p.B * p.n_groups * p.n_row_tiles * p.Hkv;
  const dim3 grid((unsigned)(units * p.n_split)), block(64 * kWaves);
  if (p.tile_rows == 32) {
    hipLaunchKernelGGL((attn_blocks_kernel<FMT, D, 1>), grid, block, 0, stream, p);
  } else {
    if constexpr (D <= 128)
      hipLaunchKernelGGL((attn_blocks_kernel<FMT, D, 2>), grid, block, 0, stream, p);
    else
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int FMT>
hipError_t launch_d(const SparseParams &p, hipStream_t stream) {
  switch (p.D) {
    case 64: return launch<FMT, 64>(p, stream);
    case 128: return launch<FMT, 128>(p, stream);
    case 256: return launch<FMT, 256>(p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace

int attn_blocks_max_slots() { return kMaxSlots; }
int attn_blocks_tile_rows(int D, int rows) { return D <= 128 && rows > 32 ? 64 : 32; }

hipError_t launch_attn_blocks(const SparseParams &p, int format, hipStream_t stream) {
  ProfileScope scope(SLOT_ATTN_BLOCKS, stream);
  switch (format) {
    case FMT_BF16: return launch_d<FMT_BF16>(p, stream);
    case FMT_MX8: return launch_d<FMT_MX8>(p, stream);
    case FMT_MX4: return launch_d<FMT_MX4>(p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace la
