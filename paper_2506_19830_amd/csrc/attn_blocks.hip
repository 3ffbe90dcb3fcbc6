// Verification attention over selected blocks of a block cache (gfx950).
//
// Every group of query tokens and KV head has a list of blocks of the prefix; its rows (tokens x query heads of the KV head)
// attend to the keys of these blocks and to the branch's own tokens up to their own:
//     out = softmax(scale q.k) v   over both,   one pass with the running maximum and sum.
//
// The products are transposed,
//     S^T (keys x rows) = K Q^T,   O^T (D x rows) += V^T P^T
// so that a lane holds scores of one row only, and P^T leaves the accumulators of the first product in the order in which
// the second one wants its operand (the keys of a tile are permuted alike on both sides).  V lies in LDS as bf16 and is read
// back transposed by 16-bit reads.  Quantised rows are widened to bf16 exactly, their exponents applied by the conversion.
// Probabilities are rounded to bf16 for the second product, at every head dimension and for fp32 results too (relative 2^-8 each
// at most, the output's own rounding where that is bf16; 2.3e-3 of a row's size from the definition, 1.7e-3 with the output's
// rounding alone): a second term would double the second product.  Scores, maxima, sums and accumulators are fp32.
//
// Two kernels.  With up to 32 rows to a group (attn_blocks_rows_kernel) the work is a stream of keys that few rows look at: every
// wavefront takes tiles of 32 keys of its own for all rows, and the wavefronts are folded at the end.  With more rows
// (attn_blocks_tile_kernel) two, three or four pairs of wavefronts with 32 rows each, one for either half of the keys, share tiles
// of 64 keys that they widen into LDS together (head dimension 256: four wavefronts and 32 keys).  Workgroups that share a
// group's keys leave partial results that the merge of long splits joins.
#include "attn_common.hpp"

namespace la {
namespace {

constexpr int kMaxSlots = 1024;  // blocks whose place a workgroup holds in LDS

typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

__device__ __forceinline__ float exp_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// Eight elements (bf16: four words, fp8: two, fp4: one) of scale s as four bf16 pairs.
template <int FMT>
__device__ __forceinline__ u32x4 widen8(const uint32_t *w, float s) {
  u32x4 x;
  if constexpr (FMT == FMT_BF16) {
    x = u32x4{w[0], w[1], w[2], w[3]};
  } else if constexpr (FMT == FMT_MX8) {
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, false));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, true));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, false));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, true));
  } else {
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 3));
  }
  return x;
}
template <int FMT>
constexpr int kWords8 = FMT == FMT_BF16 ? 4 : FMT == FMT_MX8 ? 2 : 1;

// The 16-byte pieces of a row lie permuted in LDS, piece c of key k at c ^ swizzle(k): the 16 keys that a store or a read of
// whole pieces touches at a time, and the keys x 32 or 64 bytes that one transposing read gathers, then fall evenly over the
// banks.
template <int D>
__device__ __forceinline__ int swizzle(int key) {
  return D == 64 ? (((key >> 1) & 1) << 2) | ((key >> 2) & 3) : ((key & 3) << 2) | ((key >> 2) & 3);
}

// The same where a store covers whole rows one after the other and a transposing read 16 keys x 32 bytes (attn_blocks_rows_kernel): the
// pieces of a chunk that a lane widens come one per store, so neighbouring rows differ in the lowest bits.
template <int D>
__device__ __forceinline__ int swizzle_rows(int key) {
  return D == 64 ? ((key >> 1) & 3) | (((key >> 3) & 1) << 2) : key & 15;
}

// Two transposing reads side by side: four keys of one element from each place.  (Joined as vectors of 16-bit numbers: joined
// as 32-bit words, the compiler copied every pair of registers once more.)
__device__ __forceinline__ bf16x8 read_transposed(const uint8_t *p0, const uint8_t *p1) {
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p0);
  const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p1);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// 16 bytes per lane from memory (a base the wavefront shares and an offset, or an address) to consecutive places in LDS, without
// registers in between; the wavefront that issues it waits with wait_loads() before it reads, or a barrier lets others read.
__device__ __forceinline__ void load_lds16(const uint8_t *base, uint32_t lane_off, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_off), "s"(base), "s"(lds_addr) : "m0");
}
__device__ __forceinline__ void load_lds16(const uint8_t *src, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(lds_addr) : "m0");
}
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
// Before loads are sent to a place in LDS that was read.
__device__ __forceinline__ void wait_reads() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// LDS written by some lanes is read by others of the same wavefront: the compiler must not move one across the other (the
// hardware keeps a wavefront's LDS operations in order).
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Maximum / sum over the four lanes of a row (lane, lane ^ 16, lane ^ 32, lane ^ 48).
__device__ __forceinline__ float quarter_max(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = sw[0], b = sw[1];
  return xhalf_max(fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
}
__device__ __forceinline__ float quarter_sum(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = sw[0], b = sw[1];
  return xhalf_sum(__builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
}

// What a workgroup works on.
struct Unit {
  int b, hk, tok0, n_rows, r0;  // request, KV head, first token of the group, its rows, the first one of this tile
  int split;
  int own0, own_end;            // own tokens that any row of the tile sees
  int n_keys;                   // keys of the list
  int begin, end, n_tiles;      // the workgroup's share of the unit's tiles; the first n_tiles of all are the list's
  int slot0;                    // list index of place[0]
};

struct Places {
  int32_t place[kMaxSlots];     // where the blocks lie that the workgroup's tiles come from
  int32_t last;                 // the last block listed
};

// Finds the unit's rows and keys and fills the table of places (the caller's barrier makes it visible); false: no rows.  What
// begins a workgroup is a chain of dependent loads, so everything that can be asked for at once is: a list that fits the table
// is taken whole, without waiting for its length or the prefix's.
template <int ROWS, int KEYS, int THREADS>
__device__ __forceinline__ bool find_unit(const SparseParams &p, Unit &u, Places &t) {
  // KV heads vary fastest: with eight of them each XCD keeps to one head's keys
  uint32_t id = blockIdx.x;
  u.hk = (int)(id % (uint32_t)p.Hkv);
  id /= (uint32_t)p.Hkv;
  u.split = (int)(id % (uint32_t)p.n_split);
  id /= (uint32_t)p.n_split;
  const int row_tile = (int)(id % (uint32_t)p.n_row_tiles);
  id /= (uint32_t)p.n_row_tiles;
  const int group = (int)(id % (uint32_t)p.n_groups);
  u.b = (int)(id / (uint32_t)p.n_groups);
  int n_tok = p.gamma * p.L;
  u.tok0 = 0;
  if (p.sel) {
    const int per_branch = p.n_groups / p.gamma, g = group / per_branch, t0 = (group - g * per_branch) * p.group_len;
    u.tok0 = g * p.L + t0;
    n_tok = min(p.group_len, p.L - t0);
  }
  u.n_rows = n_tok * p.G, u.r0 = row_tile * ROWS;
  if (u.r0 >= u.n_rows) return false;
  const int r_last = min(u.r0 + ROWS, u.n_rows) - 1;
  u.own0 = (u.tok0 + u.r0 / p.G) / p.L * p.L, u.own_end = u.tok0 + r_last / p.G + 1;

  const int bs = 1 << p.block_shift, tid = threadIdx.x;
  const int32_t *table = p.block_tables ? p.block_tables + (size_t)u.b * p.max_blocks : nullptr;
  auto place_of = [&](int lb) __attribute__((always_inline)) { return table ? table[lb] : u.b * p.max_blocks + lb; };
  const size_t unit = ((size_t)u.b * p.n_groups + group) * p.Hkv + u.hk;
  const int32_t *list = p.sel ? p.sel + unit * p.max_sel : nullptr;
  const bool whole = p.sel && p.max_sel <= kMaxSlots;
  constexpr int kIds = (kMaxSlots + THREADS - 1) / THREADS;
  int ids[kIds];
  if (whole) {
#pragma unroll
    for (int k = 0; k < kIds; ++k)
      if (tid + k * THREADS < p.max_sel) ids[k] = list[tid + k * THREADS];
  }
  const int listed = p.sel ? p.sel_count[unit] : 0;
  const int P = (int)min((int64_t)max(p.prefix_lens[u.b], 0), (int64_t)p.max_blocks << p.block_shift);
  const int n_blocks = (P + bs - 1) >> p.block_shift;
  u.n_keys = P;
  if (p.sel) {
    const int n = min(max(listed, 0), min(p.max_sel, n_blocks));
    int last = 0;
    if (n > 0 && whole) {
#pragma unroll
      for (int k = 0; k < kIds; ++k) {
        const int i = tid + k * THREADS, lb = min(max(ids[k], 0), n_blocks - 1);
        if (i < n) t.place[i] = place_of(lb);
        if (i == n - 1) t.last = lb;
      }
      __syncthreads();
      last = t.last;
    } else if (n > 0) {
      last = min(max(list[n - 1], 0), n_blocks - 1);
    }
    u.n_keys = n > 0 ? ((n - 1) << p.block_shift) + min(bs, P - (last << p.block_shift)) : 0;
  }
  // the unit's tiles, dealt out evenly
  u.n_tiles = (u.n_keys + KEYS - 1) / KEYS;
  const uint32_t total = (uint32_t)(u.n_tiles + (u.own_end - u.own0 + KEYS - 1) / KEYS);
  const uint32_t each = total / (uint32_t)p.n_split, more = total - each * (uint32_t)p.n_split;
  u.begin = (int)(u.split * each + min((uint32_t)u.split, more));
  u.end = u.begin + (int)(each + ((uint32_t)u.split < more ? 1u : 0u));
  u.slot0 = 0;
  if (!whole && u.begin < min(u.end, u.n_tiles)) {
    u.slot0 = (u.begin * KEYS) >> p.block_shift;
    const int slots = min(((min(u.end * KEYS, u.n_keys) - 1) >> p.block_shift) + 1 - u.slot0, kMaxSlots);
    for (int i = tid; i < slots; i += THREADS)
      t.place[i] = place_of(list ? min(max(list[u.slot0 + i], 0), n_blocks - 1) : u.slot0 + i);
  }
  return true;
}

// Where a key of the list lies: block_at its block (keys behind the last repeat it), row_at its row in the cache.
__device__ __forceinline__ int block_at(const SparseParams &p, const Unit &u, const Places &t, int key) {
  return t.place[min((min(key, u.n_keys - 1) >> p.block_shift) - u.slot0, kMaxSlots - 1)];
}
__device__ __forceinline__ size_t row_at(const SparseParams &p, const Unit &u, int blk, int key) {
  return (((size_t)(uint32_t)blk * (uint32_t)p.Hkv + (uint32_t)u.hk) << p.block_shift) + (min(key, u.n_keys - 1) & ((1 << p.block_shift) - 1));
}
// Groups of 16 keys lie in one block.  Where lanes of a wavefront share their keys' groups (attn_blocks_rows_kernel), a group's place
// goes through scalar registers, and a lane adds its offset inside the group.
struct KeyGroup {
  size_t row;   // the group's first row in the cache
  int last;     // its last key that exists (15 but at the end of the list)
};
// KEYS / 16 groups of tile `tile`, one of the workgroup's: lane l has the block of group l % (KEYS / 16)
template <int KEYS>
__device__ __forceinline__ int tile_places(const SparseParams &p, const Unit &u, const Places &t, int tile, int lane) {
  const int key = min(tile * KEYS + (lane % (KEYS / 16)) * 16, (u.n_keys - 1) & ~15);   // (groups behind the last repeat it)
  return t.place[min((key >> p.block_shift) - u.slot0, kMaxSlots - 1)];
}
template <int KEYS>
__device__ __forceinline__ KeyGroup key_group(const SparseParams &p, const Unit &u, int places, int tile, int group) {
  const int key = min(tile * KEYS + group * 16, (u.n_keys - 1) & ~15);
  const int blk = __builtin_amdgcn_readlane(places, group);
  KeyGroup g;
  g.row = (((size_t)blk * p.Hkv + u.hk) << p.block_shift) + (key & ((1 << p.block_shift) - 1));
  g.last = min(15, u.n_keys - 1 - key);
  return g;
}
// token of the request that own key `key` of a tile is (those behind the last repeat it)
__device__ __forceinline__ int own_row(const Unit &u, int first, int key) { return min(first + key, u.own_end - 1); }

__device__ __forceinline__ size_t out_row(const SparseParams &p, const Unit &u, int r) {
  return (size_t)u.b * p.n_rows + (size_t)(u.tok0 + r / p.G) * p.Hq + u.hk * p.G + r % p.G;
}

// Four consecutive results of a row: the final values, or the workgroup's partial.
__device__ __forceinline__ void put_out(const SparseParams &p, const Unit &u, size_t grow, int d, int D, f32x4 x, float inv) {
  if (p.part_o) {
    *(f32x4 *)(p.part_o + ((size_t)u.split * p.B * p.n_rows + grow) * D + d) = x;
  } else if (p.out_f32) {
    *(f32x4 *)((float *)p.out + grow * D + d) = x * inv;
  } else {
    x *= inv;
    *(u32x2 *)((uint8_t *)p.out + (grow * D + d) * 2) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  }
}
__device__ __forceinline__ void put_sums(const SparseParams &p, const Unit &u, size_t grow, float m, float l) {
  if (p.part_o)
    *(f32x2 *)(p.part_ml + ((size_t)u.split * p.B * p.n_rows + grow) * 2) = f32x2{m, l};
  else if (p.lse)
    p.lse[grow] = 0.69314718055994530942f * (m + __builtin_log2f(l));
}

enum TileMask { TILE_FULL = 0, TILE_TAIL, TILE_OWN };

// ---------------------------------------------------------------------------------------------------- few rows

// A quarter of one key's row, as stored: elements q D/4 .. of quarter q.
template <int FMT, int D>
struct Quarter {
  static constexpr int kWords = D / 32 * kWords8<FMT>;
  uint32_t w[kWords];
  uint32_t e;  // the aligned word of exponents that holds those of its group (D = 256: of its two groups)
};
// (A word, and the byte taken out of it at its use: bytes were widened to registers right behind the loads, which waited for
// memory in every tile.)
template <int D>
__device__ __forceinline__ int exp_shift(size_t row, int q) { return (int)((row * (D / 32) + q * D / 128) & 3) * 8; }

// base, exps: row 0 of a group (the same for all lanes); at: the lane's row in it
template <int FMT, int D>
__device__ __forceinline__ void load_quarter(Quarter<FMT, D> &r, const uint8_t *base, const uint8_t *exps, uint32_t at, int q) {
  constexpr int N = Quarter<FMT, D>::kWords;
  const uint32_t off = at * (16 * N) + q * (N * 4);
  if constexpr (N == 2) {
    const u32x2 x = *(const u32x2 *)(base + off);
    r.w[0] = x[0], r.w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = *(const u32x4 *)(base + off + i * 4);
      r.w[i] = x[0], r.w[i + 1] = x[1], r.w[i + 2] = x[2], r.w[i + 3] = x[3];
    }
  }
  if constexpr (FMT != FMT_BF16) r.e = *(const uint32_t *)(exps + ((at * (D / 32) + q * D / 128) & ~3u));
}

// shift: of the first group's exponent in its word
template <int FMT, int D>
__device__ __forceinline__ u32x4 widen(const Quarter<FMT, D> &r, int t, int shift) {
  return widen8<FMT>(r.w + t * kWords8<FMT>, FMT == FMT_BF16 ? 0.f : exp_scale((r.e >> (shift + 8 * (t / 4))) & 0xffu));
}

template <int D, int RB>
struct Rows {
  bf16x8 q[RB][D / 32];        // row n of block rb: elements quarter (D / 4) + 8 t ..
  f32x4 o[RB][D / 16];         // O^T: row n, d = 16 db + 4 quarter + 0..3
  float m[RB], l[RB];          // running maximum (log2 units) and this lane's share of the sum
  int tok[RB], start[RB];      // token of the row inside the request, first token of its branch
};

// Scores of the 32 keys of a tile, probabilities, and the product with the V tile in LDS.  first: the tile's first key; keys
// from `limit` on do not exist (TILE_TAIL).
template <int D, int RB, int MASK>
__device__ __forceinline__ void attend_rows(Rows<D, RB> &st, f32x4 (&s)[RB][2], const uint8_t *lds, int vt_read, float scale_log2, int first,
                                            int limit, int lane) {
  const int quarter = lane >> 4;
  float alpha[RB];
  bool raise = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = first + 16 * u + 4 * quarter + j;
        if constexpr (MASK == TILE_TAIL) {
          if (key >= limit) s[rb][u][j] = -INFINITY;
        } else if constexpr (MASK == TILE_OWN) {
          if (key > st.tok[rb] || key < st.start[rb]) s[rb][u][j] = -INFINITY;
        }
        top = fmaxf(top, s[rb][u][j]);
      }
    top = quarter_max(top) * scale_log2;
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
      for (int db = 0; db < D / 16; ++db) st.o[rb][db] *= alpha[rb];
    }
  }
  // V^T operands: lane (d, quarter) takes keys 4 quarter + 0..3 and 16 more, the order of the probabilities.  A batch is read
  // while the exponentials run, the next one while the matrix cores work on it.
  constexpr int kBatch = 4;
  bf16x8 vf[2][kBatch];
  auto read_batch = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < kBatch; ++db) {
      const uint8_t *at = lds + (vt_read ^ ((i * kBatch + db) << 5));
      vf[i & 1][db] = read_transposed(at, at + 16 * D * 2);
    }
  };
  read_batch(0);
  __builtin_amdgcn_sched_barrier(0);
  bf16x8 pf[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float base = st.m[rb] == -INFINITY ? 0.f : st.m[rb];  // no key seen yet: every score is -inf
    float sum = 0.f;
    u32x4 w;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][u][j], scale_log2, -base));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][u][j + 1], scale_log2, -base));
        sum += p0 + p1;
        w[2 * u + j / 2] = pack_bf16(p0, p1);
      }
    pf[rb] = __builtin_bit_cast(bf16x8, w);
    st.l[rb] += sum;
  }
#pragma unroll
  for (int i = 0; i < D / 16 / kBatch; ++i) {
    if (i + 1 < D / 16 / kBatch) {
      read_batch(i + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int db = 0; db < kBatch; ++db)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        st.o[rb][i * kBatch + db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i & 1][db], pf[rb], st.o[rb][i * kBatch + db], 0, 0, 0);
  }
}

// (u: which 16 of the tile's 32 keys)
template <int FMT, int D, int RB>
__device__ __forceinline__ void scores_rows(f32x4 (&s)[RB][2], int u, const Quarter<FMT, D> &k, int shift, const Rows<D, RB> &st) {
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) s[rb][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < D / 32; ++t) {
    const bf16x8 kf = __builtin_bit_cast(bf16x8, widen<FMT, D>(k, t, shift));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, st.q[rb][t], s[rb][u], 0, 0, 0);
  }
}

template <int FMT, int D>
__device__ __forceinline__ void stage_rows(uint8_t *lds, int vt_write, int u, const Quarter<FMT, D> &v, int shift) {
#pragma unroll
  for (int t = 0; t < D / 32; ++t) *(u32x4 *)(lds + (vt_write ^ (t << 4)) + u * 16 * D * 2) = widen<FMT, D>(v, t, shift);
}

// A tile of 32 keys on its way to one wavefront.  The tag look-ups of the cache are what such a stream can be bound by: a load
// whose neighbouring lanes read different rows takes one for every lane, one whose lanes read whole rows one for 64 bytes or
// more.  V comes in whole rows, through registers, and goes to LDS as bf16.  K wants a row for every lane: quantised, a lane's
// quarter of a row is one or two loads, which is cheaper than a way through LDS (32 requests x 32 blocks, fp4: 17.2 us, through
// LDS 20.9; 54 groups of 5 rows, fp8: 26.4 us and 28.6; V and K both a row for every lane: 17.1 and 36.6); as
// bf16 it is four, and K goes through LDS as stored (48 requests: 79 us and 105).  There the pieces of a row lie permuted: piece
// c of key k at c ^ key_mix(k), so that one piece of 16 keys misses no bank.
template <int FMT, int D>
struct Stream {
  static constexpr int kRowBytes = FMT == FMT_BF16 ? 2 * D : FMT == FMT_MX8 ? D : D / 2;
  static constexpr int kChunks = kRowBytes / 16, kElems = D / kChunks;   // of a row; elements of a chunk
  static constexpr int kLoads = kChunks / 2, kRows = 64 / kChunks;        // of a tensor's tile; rows of a load
  static constexpr bool kStaged = FMT == FMT_BF16;                        // K goes through LDS
  static constexpr int kKeyBytes = kStaged ? 32 * kRowBytes : 0;
  u32x4 v[kLoads];
  uint32_t ve[kLoads];
  Quarter<FMT, D> k[2];
  static __device__ __forceinline__ int key_mix(int key) { return kChunks < 16 ? (key * kChunks / 16) & (kChunks - 1) : key & 15; }
};

// k_lds: the wavefront's place for K.  group_of(x): keys 16 x .. of the tile.
template <int FMT, int D, typename F>
__device__ __forceinline__ void stream_load(Stream<FMT, D> &g, uint32_t k_lds, const SparseParams &p, int lane, F group_of) {
  using S = Stream<FMT, D>;
  const KeyGroup kg[2] = {group_of(0), group_of(1)};
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int key = i * S::kRows + lane / S::kChunks, chunk = lane % S::kChunks;
    // (where a row has two chunks a load is all 32 keys, otherwise its keys are of one group)
    const bool upper = S::kRows > 16 ? lane >= 32 : i * S::kRows >= 16;
    const size_t first = upper ? kg[1].row : kg[0].row;
    const uint32_t at = (uint32_t)min(key & 15, upper ? kg[1].last : kg[0].last), off = at * S::kRowBytes;
    if constexpr (S::kStaged) load_lds16((const uint8_t *)p.k_cache + first * S::kRowBytes, off + (chunk ^ S::key_mix(key)) * 16, k_lds + i * 1024);
    g.v[i] = *(const u32x4 *)((const uint8_t *)p.v_cache + first * S::kRowBytes + off + chunk * 16);
    if constexpr (FMT != FMT_BF16) g.ve[i] = *(const uint32_t *)(p.v_exp + first * (D / 32) + ((at * (D / 32) + chunk * S::kElems / 32) & ~3u));
  }
  if constexpr (!S::kStaged) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
      load_quarter(g.k[x], (const uint8_t *)p.k_cache + kg[x].row * S::kRowBytes, p.k_exp + kg[x].row * (D / 32), (uint32_t)min(lane & 15, kg[x].last),
                   lane >> 4);
  }
}

// V into its place.  last: the tile's last key that exists.  (A block's rows begin at a multiple of 16, so the key says where in
// its word an exponent is.)
template <int FMT, int D>
__device__ __forceinline__ void stream_values(const Stream<FMT, D> &g, uint8_t *v_lds, int last, int lane) {
  using S = Stream<FMT, D>;
  constexpr int kPieces = S::kElems / 8;
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int key = i * S::kRows + lane / S::kChunks, chunk = lane % S::kChunks;
    const int row = key * D * 2 + (((chunk * kPieces) ^ swizzle_rows<D>(key)) << 4);
    const uint32_t w[4] = {g.v[i][0], g.v[i][1], g.v[i][2], g.v[i][3]};
    float scale = 0.f;
    if constexpr (FMT != FMT_BF16) scale = exp_scale((g.ve[i] >> (((min(key, last) * (D / 32) + chunk * S::kElems / 32) & 3) * 8)) & 0xffu);
#pragma unroll
    for (int t = 0; t < kPieces; ++t) *(u32x4 *)(v_lds + (row ^ (t << 4))) = widen8<FMT>(w + t * kWords8<FMT>, scale);
  }
}

// The lane's quarter of key n of group x, out of LDS.
template <int D>
__device__ __forceinline__ void staged_quarter(Quarter<FMT_BF16, D> &r, const uint8_t *k_lds, int x, int lane) {
  using S = Stream<FMT_BF16, D>;
  const int key = x * 16 + (lane & 15), first = (lane >> 4) * (S::kChunks / 4);
#pragma unroll
  for (int i = 0; i < S::kChunks / 4; ++i) {
    const u32x4 w = *(const u32x4 *)(k_lds + key * S::kRowBytes + (((first + i) ^ S::key_mix(key)) << 4));
    r.w[4 * i] = w[0], r.w[4 * i + 1] = w[1], r.w[4 * i + 2] = w[2], r.w[4 * i + 3] = w[3];
  }
}

// Wavefronts of a SIMD that the registers are allotted for: a wavefront alone issues a vector instruction about every other
// time it could, so as many as the accumulators, and with bf16 the tiles in LDS, leave room for.
template <int FMT, int D, int RB>
constexpr int kRowsOccupancy = D == 256 ? (RB == 1 && FMT != FMT_BF16 ? 2 : 1) : D == 128 ? (RB == 1 && FMT != FMT_BF16 ? 3 : 2) : RB == 2 ? 2 : 4;

// RB blocks of 16 rows, NW wavefronts with tiles of their own.  Bound by the stream of keys where it is long (fp4, 32 requests x 8
// heads x 2048 keys: 17.2 us, 4.2 TB/s; fp8, 8 prefixes of 8K to 32K keys: 70 us, 4.3 TB/s), by conversions and cache reads where
// groups share the keys (fp8, 54 groups x 8 heads x 2048 keys: 28.4 us, 26.4 among other calls).
template <int FMT, int D, int RB, int NW>
__global__ __launch_bounds__(64 * NW, (kRowsOccupancy<FMT, D, RB>)) void attn_blocks_rows_kernel(const SparseParams p) {
  constexpr int kTileBytes = 32 * D * 2;            // V tile of a wavefront
  constexpr int kKeyBytes = Stream<FMT, D>::kKeyBytes;   // its K tile, as stored
  constexpr int kOne = RB * (D / 16) * 4 * 64;      // floats of one wavefront's accumulators
  constexpr int kTiles = NW * (kTileBytes + kKeyBytes), kBytes = kTiles > NW / 2 * kOne * 4 ? kTiles : NW / 2 * kOne * 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kBytes];
  __shared__ Places places;
  __shared__ float fold_ml[NW][RB * 16][2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, quarter = lane >> 4;
  Unit u;
  if (!find_unit<RB * 16, 32, 64 * NW>(p, u, places)) return;
  const int n_tiles = u.n_tiles;
  const int each = (u.end - u.begin) / NW, more = (u.end - u.begin) % NW;
  const int begin = u.begin + wave * each + min(wave, more), end = begin + each + (wave < more ? 1 : 0);

  Rows<D, RB> st;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = min(u.r0 + rb * 16 + n, u.n_rows - 1);
    const int tok = u.tok0 + r / p.G;
    const uint8_t *src = (const uint8_t *)p.q + out_row(p, u, r) * D * 2 + quarter * (D / 2);
#pragma unroll
    for (int t = 0; t < D / 32; ++t) st.q[rb][t] = *(const bf16x8 *)(src + t * 16);
    st.tok[rb] = tok, st.start[rb] = tok / p.L * p.L;
    st.m[rb] = -INFINITY, st.l[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) st.o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();

  // offsets into LDS (a row's pieces are permuted inside the row, whose size is a power of two: pieces are reached by XOR)
  const int vt_write = wave * kTileBytes + n * D * 2 + (((quarter * (D / 32)) ^ swizzle_rows<D>(n)) << 4);
  const int read_key = 4 * quarter + (n >> 2);
  const int vt_read = wave * kTileBytes + read_key * D * 2 + ((((n & 3) >> 1) ^ swizzle_rows<D>(read_key)) << 4) + (n & 1) * 8;
  // the prefix: the rows of the next tile are requested before the present one is used
  const int pre_end = min(end, n_tiles);
  if (begin < pre_end) {
    // A tile is requested anew as soon as the scores and the V tile of the one before are made; the scheduling fence keeps the
    // compiler from moving the requests down to where the next tile needs them.
    Stream<FMT, D> g;
    uint8_t *k_lds = lds + NW * kTileBytes + wave * kKeyBytes;
    int at_places = tile_places<32>(p, u, places, begin, lane);
    auto request = [&](int tile) __attribute__((always_inline)) {
      const int pl = at_places;
      at_places = tile_places<32>(p, u, places, min(tile + 1, pre_end - 1), lane);   // (the table ends with the workgroup's tiles)
      stream_load(g, lds_address(k_lds), p, lane, [&](int x) __attribute__((always_inline)) { return key_group<32>(p, u, pl, tile, x); });
    };
    auto consume = [&](f32x4 (&s)[RB][2], int last) __attribute__((always_inline)) {
      if constexpr (Stream<FMT, D>::kStaged) wait_loads();
      stream_values(g, lds + wave * kTileBytes, last, lane);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if constexpr (Stream<FMT, D>::kStaged) staged_quarter(g.k[x], k_lds, x, lane);
        scores_rows(s, x, g.k[x], exp_shift<D>((size_t)min(x * 16 + n, last), quarter), st);
      }
      if constexpr (Stream<FMT, D>::kStaged) wait_reads();
    };
    request(begin);
    const int full_end = min(pre_end, u.n_keys / 32);   // (only the list's last tile can be a partial one)
    for (int tile = begin; tile < full_end; ++tile) {
      f32x4 s[RB][2];
      consume(s, 31);
      if (tile + 1 < pre_end) request(tile + 1);
      __builtin_amdgcn_sched_barrier(0);
      wave_order();
      attend_rows<D, RB, TILE_FULL>(st, s, lds, vt_read, p.scale_log2, tile * 32, u.n_keys, lane);
      wave_order();
    }
    if (full_end < pre_end) {
      f32x4 s[RB][2];
      consume(s, u.n_keys - 1 - full_end * 32);
      wave_order();
      attend_rows<D, RB, TILE_TAIL>(st, s, lds, vt_read, p.scale_log2, full_end * 32, u.n_keys, lane);
      wave_order();
    }
  }
  // the branch's own tokens
  for (int tile = max(begin, n_tiles); tile < end; ++tile) {
    const int first = u.own0 + (tile - n_tiles) * 32;
    f32x4 s[RB][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const size_t row = (((size_t)u.b * p.gamma * p.L + own_row(u, first, x * 16 + n)) * p.Hkv + u.hk) * D * 2;
      Quarter<FMT_BF16, D> r;
      load_quarter(r, (const uint8_t *)p.v_branch + row, nullptr, 0, quarter);
      stage_rows(lds, vt_write, x, r, 0);
      wave_order();   // (one half row in registers at a time)
      load_quarter(r, (const uint8_t *)p.k_branch + row, nullptr, 0, quarter);
      scores_rows(s, x, r, 0, st);
      wave_order();
    }
    attend_rows<D, RB, TILE_OWN>(st, s, lds, vt_read, p.scale_log2, first, u.own_end, lane);
    wave_order();
  }

  // fold the wavefronts: common maximum, then the accumulators through LDS, half of those left at a time
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    st.l[rb] = quarter_sum(st.l[rb]);
    if (quarter == 0) fold_ml[wave][rb * 16 + n][0] = st.m[rb], fold_ml[wave][rb * 16 + n][1] = st.l[rb];
  }
  __syncthreads();  // (also: every wavefront is done with its V tile)
  float m_all[RB], l_all[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_all[rb] = -INFINITY, l_all[rb] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) m_all[rb] = fmaxf(m_all[rb], fold_ml[w][rb * 16 + n][0]);
    const float base = m_all[rb] == -INFINITY ? 0.f : m_all[rb];
#pragma unroll
    for (int w = 0; w < NW; ++w)
      l_all[rb] += fold_ml[w][rb * 16 + n][1] * __builtin_amdgcn_exp2f(fold_ml[w][rb * 16 + n][0] - base);
    const float f = __builtin_amdgcn_exp2f(st.m[rb] - base);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) st.o[rb][db] *= f;
  }
  f32x4 *buf = (f32x4 *)lds;
#pragma unroll
  for (int left = NW; left > 1; left /= 2) {
    if (wave >= left / 2 && wave < left) {
      f32x4 *dst = buf + (wave - left / 2) * (kOne / 4) + lane;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int db = 0; db < D / 16; ++db) dst[(rb * (D / 16) + db) * 64] = st.o[rb][db];
    }
    __syncthreads();
    if (wave < left / 2) {
      const f32x4 *src = buf + wave * (kOne / 4) + lane;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int db = 0; db < D / 16; ++db) st.o[rb][db] += src[(rb * (D / 16) + db) * 64];
    }
    if (left > 2) __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = u.r0 + rb * 16 + n;
    if (r >= u.n_rows) continue;
    const size_t grow = out_row(p, u, r);
    if (quarter == 0) put_sums(p, u, grow, m_all[rb], l_all[rb]);
    const float inv = 1.0f / l_all[rb];
#pragma unroll
    for (int db = 0; db < D / 16; ++db) put_out(p, u, grow, db * 16 + quarter * 4, D, st.o[rb][db], inv);
  }
}

// ---------------------------------------------------------------------------------------------------- many rows

// A tile on its way from memory to LDS, K and V as wavefront loads of 64 x 16 bytes that the NW wavefronts of the workgroup take
// in turn.  Quantised rows pass through registers: lane (key n of 16, chunk quarter + 4 i), so that one load takes whole rows
// of 64 bytes and more, and one store instruction one piece of 16 keys.  bf16 rows go to LDS at once: lane l of a load fills
// place l of 64 pieces, so it fetches the piece that belongs there.
template <int FMT, int D, int KEYS, int NW>
struct Stage {
  static constexpr int kElems = FMT == FMT_BF16 ? 8 : FMT == FMT_MX8 ? 16 : 32;   // of 16 bytes
  static constexpr int kChunks = D / kElems;                                      // of a row
  static constexpr int kGroups = kChunks < 4 ? 1 : kChunks / 4;                   // wavefront loads per 16 keys
  static constexpr int kTensor = FMT == FMT_BF16 ? KEYS * kChunks / 64 : KEYS / 16 * kGroups;   // of K, and of V
  static constexpr int kLoads = (2 * kTensor + NW - 1) / NW;
  // a wavefront's loads of V are those of K a tile earlier: their rows need not be found again
  static constexpr bool kAgain = kTensor % NW == 0;
  u32x4 w[FMT == FMT_BF16 ? 1 : kLoads];
  uint32_t e[FMT == FMT_BF16 ? 1 : kLoads];
};

// The key of a tile that a lane fetches (a piece of) by load `at` of a tensor.
template <int FMT, int D, int KEYS, int NW>
__device__ __forceinline__ int stage_key(int at, int lane) {
  using S = Stage<FMT, D, KEYS, NW>;
  return FMT == FMT_BF16 ? (at * 64 + lane) / S::kChunks : at / S::kGroups * 16 + (lane & 15);
}

// row_of(i): the row for load i; kt, vt: the tiles' places in LDS (bf16)
template <int FMT, int D, int KEYS, int NW, typename F>
__device__ __forceinline__ void stage_load(Stage<FMT, D, KEYS, NW> &g, const uint8_t *kt, const uint8_t *vt, const void *kb, const void *vb,
                                           const uint8_t *kx, const uint8_t *vx, F row_of) {
  using S = Stage<FMT, D, KEYS, NW>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int load = wave + i * NW, which = load >= S::kTensor ? 1 : 0, at = load - which * S::kTensor;
    if (load >= 2 * S::kTensor) continue;
    const uint8_t *base = (const uint8_t *)(which ? vb : kb);
    const size_t row = row_of(i);
    if constexpr (FMT == FMT_BF16) {
      const int chunk = (lane % S::kChunks) ^ swizzle<D>(stage_key<FMT, D, KEYS, NW>(at, lane));
      load_lds16(base + (row * S::kChunks + chunk) * 16, lds_address(which ? vt : kt) + at * 1024);
    } else {
      const int chunk = min((lane >> 4) + 4 * (at % S::kGroups), S::kChunks - 1);
      g.w[i] = *(const u32x4 *)(base + (row * S::kChunks + chunk) * 16);
      g.e[i] = *(const uint32_t *)((which ? vx : kx) + ((row * (D / 32) + chunk * S::kElems / 32) & ~(size_t)3));
    }
  }
}

// Before the barrier behind which the tiles are read.  k_last, v_last: the last key of each that exists (those behind it repeat
// it).
template <int FMT, int D, int KEYS, int NW>
__device__ __forceinline__ void stage_store(const Stage<FMT, D, KEYS, NW> &g, uint8_t *kt, uint8_t *vt, int k_last, int v_last) {
  using S = Stage<FMT, D, KEYS, NW>;
  if constexpr (FMT == FMT_BF16) {
    wait_loads();
  } else {
    constexpr int kPieces = S::kElems / 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int load = wave + i * NW, which = load >= S::kTensor ? 1 : 0, at = load - which * S::kTensor;
      if (load >= 2 * S::kTensor) continue;
      const int key = at / S::kGroups * 16 + (lane & 15), chunk = (lane >> 4) + 4 * (at % S::kGroups);
      if (S::kChunks < 4 && chunk >= S::kChunks) continue;   // (a D = 64 row of fp4 has two chunks)
      const uint32_t w[4] = {g.w[i][0], g.w[i][1], g.w[i][2], g.w[i][3]};
      // (a block's rows begin at a multiple of 16, so the key says where in its word an exponent is)
      const uint32_t e = (g.e[i] >> (((min(key, which ? v_last : k_last) * (D / 32) + chunk * S::kElems / 32) & 3) * 8)) & 0xffu;
      const int row = key * D * 2 + (((chunk * kPieces) ^ swizzle<D>(key)) << 4);
      uint8_t *to = which ? vt : kt;
#pragma unroll
      for (int t = 0; t < kPieces; ++t) *(u32x4 *)(to + (row ^ (t << 4))) = widen8<FMT>(w + t * kWords8<FMT>, exp_scale(e));
    }
  }
}

template <int D>
struct TileRows {
  bf16x8 q[D / 16];            // row ln: d = 16 t + 8 h ..
  f32x16 o[D / 32];
  float m, l;
  int tok, start;
};

// A wavefront's NB blocks of 32 keys of a tile.  kt, vt: offsets of the lane's K and V operands in LDS.
template <int D, int NB>
__device__ __forceinline__ void tile_scores(f32x16 (&s)[NB], const TileRows<D> &st, const uint8_t *lds, int kt) {
#pragma unroll
  for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
    for (int j = 0; j < 16; ++j) s[kb][j] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      const bf16x8 kf = *(const bf16x8 *)(lds + (kt ^ (t << 5)) + kb * 32 * D * 2);
      s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, st.q[t], s[kb], 0, 0, 0);
    }
  }
}

// Masks, and the running maximum (raised only when a tile exceeds it by kRaise: until then probabilities may reach 2^kRaise).
// first: the first key; keys from `limit` on do not exist (TILE_TAIL).
template <int D, int NB, int MASK>
__device__ __forceinline__ void tile_max(f32x16 (&s)[NB], TileRows<D> &st, float scale_log2, int first, int limit, int h) {
  float top = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int key = first + kb * 32 + (j >> 2) * 8 + h * 4 + (j & 3);
      if constexpr (MASK == TILE_TAIL) {
        if (key >= limit) s[kb][j] = -INFINITY;
      } else if constexpr (MASK == TILE_OWN) {
        if (key > st.tok || key < st.start) s[kb][j] = -INFINITY;
      }
      top = fmaxf(top, s[kb][j]);
    }
  top = xhalf_max(top) * scale_log2;
  const bool up = top > st.m + kRaise;
  const float m = up ? top : st.m;
  if (__builtin_amdgcn_ballot_w64(up)) {
    const float alpha = up ? __builtin_amdgcn_exp2f(st.m - m) : 1.0f;
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) st.o[db][j] *= alpha;
  }
  st.m = m;
}

// Probabilities of a block of 32 keys and their sum.
template <int D>
__device__ __forceinline__ void tile_probs(bf16x8 (&pf)[2], const f32x16 &s, TileRows<D> &st, float scale_log2) {
  const float base = st.m == -INFINITY ? 0.f : st.m;  // no key seen yet: every score is -inf
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    u32x4 pw;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * c + 2 * x], scale_log2, -base));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * c + 2 * x + 1], scale_log2, -base));
      sum += p0 + p1;
      pw[x] = pack_bf16(p0, p1);
    }
    pf[c] = __builtin_bit_cast(bf16x8, pw);
  }
  st.l += sum;
}

// V^T operands: lane (d, h) takes keys 16 c + 4 h + 0..3 and 8 more, the order of the probabilities.
template <int D>
__device__ __forceinline__ void tile_values(TileRows<D> &st, const bf16x8 (&pf)[2], const uint8_t *lds, int vt) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const uint8_t *at = lds + 16 * c * D * 2;
      const bf16x8 vf = read_transposed(at + (vt ^ (db << 6)), at + (vt ^ (db << 6) ^ 32) + 8 * D * 2);
      st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[c], st.o[db], 0, 0, 0);
    }
}

// 2^x at this place of the instruction stream: the compiler would gather the exponentials of a step behind its matrix
// instructions.  (The wait state lies between a transcendental instruction and what reads its result.)
__device__ __forceinline__ float exp2_here(float x) {
  float y;
  asm volatile("v_exp_f32 %0, %1\n\ts_nop 0" : "=v"(y) : "v"(x));
  return y;
}

// One block of 32 keys' probabilities and product with V, and the scores of the block that comes next: the matrix cores form
// these while the exponentials run.  The order is written out -- a matrix instruction, the vector work of two probabilities, the
// reads of operands that are needed later -- and fenced, or the compiler would put each kind of work in a row of its own.
template <int D>
__device__ __forceinline__ void tile_step(f32x16 &next, const f32x16 &s, TileRows<D> &st, const uint8_t *k_lds, int kt, const uint8_t *v_lds, int vt,
                                          float scale_log2) {
  constexpr int T = D / 16, kAhead = 4, kEach = 16 / T;  // matrix instructions; K operands under way; probabilities between two of them
  static_assert(T >= kAhead && 16 % T == 0, "head dimensions 64, 128 and 256");
  const float base = st.m == -INFINITY ? 0.f : st.m;  // no key seen yet: every score is -inf
  auto read_k = [&](int t) __attribute__((always_inline)) { return *(const bf16x8 *)(k_lds + (kt ^ (t << 5))); };
  bf16x8 kf[T], vf[T];
  float pr[16], sum = 0.f;
#pragma unroll
  for (int t = 0; t < kAhead; ++t) kf[t] = read_k(t);
#pragma unroll
  for (int j = 0; j < 16; ++j) next[j] = 0.f;
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int t = 0; t < T; ++t) {
    if (t + kAhead < T) kf[t + kAhead] = read_k(t + kAhead);
    // V operand t: keys 16 c .., elements 32 db ..
    const int c = t / (D / 32), db = t % (D / 32);
    const uint8_t *at = v_lds + 16 * c * D * 2;
    vf[t] = read_transposed(at + (vt ^ (db << 6)), at + (vt ^ (db << 6) ^ 32) + 8 * D * 2);
    next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t], st.q[t], next, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = t * kEach; j < (t + 1) * kEach; ++j) pr[j] = exp2_here(__builtin_fmaf(s[j], scale_log2, -base));
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) sum += pr[j];
  st.l += sum;
  bf16x8 pf[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    u32x4 pw;
#pragma unroll
    for (int x = 0; x < 4; ++x) pw[x] = pack_bf16(pr[8 * c + 2 * x], pr[8 * c + 2 * x + 1]);
    pf[c] = __builtin_bit_cast(bf16x8, pw);
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
    st.o[t % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t], pf[t / (D / 32)], st.o[t % (D / 32)], 0, 0, 0);
}

// RW wavefronts side by side along the rows, KS along the keys of a tile.  LDS reads, exponentials and matrix instructions of a
// step each take about a third of its time and overlap in part only: 320 rows x 64 groups x 2048 keys, bf16, 96 rows to a
// workgroup: 53 us among other calls, 415 TFLOP/s (scores, exponentials and values one after the other: 55), 58 alone.
template <int FMT, int D, int RW, int KS>
__global__ __launch_bounds__(64 * RW * KS, D == 256 ? 1 : 2) void attn_blocks_tile_kernel(const SparseParams p) {
  constexpr int KEYS = D == 256 ? 32 : 64, NB = KEYS / 32 / KS, NW = RW * KS;
  static_assert(NB == 1, "every wavefront has 32 keys of a tile");
  constexpr int kTileBytes = KEYS * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t lds[4 * kTileBytes];  // two buffers of a K and a V tile
  __shared__ Places places;
  __shared__ float fold_ml[RW * 32][2];
  static_assert(KS == 1 || RW * (D / 32) * 16 * 64 * 4 <= 4 * kTileBytes, "the accumulators of the upper keys fit");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane & 31, h = lane >> 5;
  const int row_wave = wave % RW, key_wave = wave / RW;
  Unit u;
  if (!find_unit<RW * 32, KEYS, 64 * NW>(p, u, places)) return;
  const int n_tiles = u.n_tiles, begin = u.begin, end = u.end, pre_end = min(end, n_tiles);

  TileRows<D> st;
  const int r = u.r0 + row_wave * 32 + ln, r_in = min(r, u.n_rows - 1);
  {
    const uint8_t *src = (const uint8_t *)p.q + out_row(p, u, r_in) * D * 2 + h * 16;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) st.q[t] = *(const bf16x8 *)(src + t * 32);
    st.tok = u.tok0 + r_in / p.G, st.start = st.tok / p.L * p.L;
    st.m = -INFINITY, st.l = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) st.o[db][j] = 0.f;
  }
  // the lane's operands in a buffer (a row's pieces are permuted inside the row, whose size is a power of two: XOR)
  const int i = lane & 15, read_key = 4 * h + (i >> 2), my_keys = key_wave * NB * 32;
  const int kt = (my_keys + ln) * D * 2 + ((h ^ swizzle<D>(ln)) << 4);
  const int vt = (my_keys + read_key) * D * 2 + (((2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) ^ swizzle<D>(read_key)) << 4) + (i & 1) * 8;
  uint8_t *k_lds = lds, *v_lds = lds + 2 * kTileBytes;  // two K tiles, two V tiles
  __syncthreads();

  // The prefix.  While the probabilities and the values of one tile are worked on, the matrix cores already form the next one's
  // scores: a step needs the V tile of its own and the K tile of the next, and requests the K tile behind that and the next V.
  if (begin < pre_end) {
    Stage<FMT, D, KEYS, NW> g;
    using S = Stage<FMT, D, KEYS, NW>;
    // Tiles behind the last one repeat it.  (v_tile is the last request's k_tile.)  The table of places is read a tile ahead.
    constexpr int kRows = S::kAgain ? S::kTensor / NW : S::kLoads;
    size_t row[kRows], row_before[kRows];
    int blk[kRows];
    auto key_of = [&](int i, int k_tile, int v_tile) __attribute__((always_inline)) {
      const int load = wave + i * NW, which = load >= S::kTensor ? 1 : 0;
      return min(which ? v_tile : k_tile, pre_end - 1) * KEYS + stage_key<FMT, D, KEYS, NW>(load - which * S::kTensor, lane);
    };
#pragma unroll
    for (int i = 0; i < kRows; ++i) blk[i] = block_at(p, u, places, key_of(i, begin, begin)), row[i] = 0;
    auto request = [&](int k_tile, int v_tile) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        row_before[i] = row[i], row[i] = row_at(p, u, blk[i], key_of(i, k_tile, v_tile));
        blk[i] = block_at(p, u, places, key_of(i, k_tile + 1, k_tile));
      }
      stage_load(g, k_lds + (k_tile & 1) * kTileBytes, v_lds + (v_tile & 1) * kTileBytes, p.k_cache, p.v_cache, p.k_exp, p.v_exp,
                 [&](int i) __attribute__((always_inline)) { return i < kRows ? row[i] : row_before[i % kRows]; });
    };
    auto deliver = [&](int k_tile, int v_tile) __attribute__((always_inline)) {
      stage_store(g, k_lds + (k_tile & 1) * kTileBytes, v_lds + (v_tile & 1) * kTileBytes,
                  u.n_keys - 1 - min(k_tile, pre_end - 1) * KEYS, u.n_keys - 1 - min(v_tile, pre_end - 1) * KEYS);
    };
    request(begin, begin);   // (of V nothing that is used)
    deliver(begin, begin);
    request(begin + 1, begin);
    __syncthreads();
    f32x16 s[NB];
    tile_scores(s, st, k_lds + (begin & 1) * kTileBytes, kt);
    if ((begin + 1) * KEYS <= u.n_keys)
      tile_max<D, NB, TILE_FULL>(s, st, p.scale_log2, begin * KEYS + my_keys, u.n_keys, h);
    else
      tile_max<D, NB, TILE_TAIL>(s, st, p.scale_log2, begin * KEYS + my_keys, u.n_keys, h);
    deliver(begin + 1, begin);
    __syncthreads();
    auto weigh = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        bf16x8 pf[2];
        tile_probs(pf, s[kb], st, p.scale_log2);
        tile_values(st, pf, v_lds + (tile & 1) * kTileBytes + kb * 32 * D * 2, vt);
      }
    };
    const int full_end = min(pre_end, u.n_keys / KEYS);   // (only the list's last tile can be a partial one)
    int tile = begin;
    for (; tile + 1 < full_end; ++tile) {
      request(tile + 2, tile + 1);
      f32x16 next[1];
      tile_step<D>(next[0], s[0], st, k_lds + ((tile + 1) & 1) * kTileBytes, kt, v_lds + (tile & 1) * kTileBytes, vt, p.scale_log2);
      tile_max<D, 1, TILE_FULL>(next, st, p.scale_log2, (tile + 1) * KEYS + my_keys, u.n_keys, h);
      s[0] = next[0];
      deliver(tile + 2, tile + 1);
      __syncthreads();
    }
    if (tile + 1 < pre_end) {
      request(tile + 2, tile + 1);
      weigh(tile);
      tile_scores(s, st, k_lds + ((tile + 1) & 1) * kTileBytes, kt);
      tile_max<D, NB, TILE_TAIL>(s, st, p.scale_log2, (tile + 1) * KEYS + my_keys, u.n_keys, h);
      deliver(tile + 2, tile + 1);
      __syncthreads();
    }
    weigh(pre_end - 1);
    __syncthreads();
  }
  // the branches' own tokens
  for (int tile = max(begin, n_tiles); tile < end; ++tile) {
    const int first = u.own0 + (tile - n_tiles) * KEYS;
    constexpr int kPieces = D / 8;
    for (int load = __builtin_amdgcn_readfirstlane(wave); load < 2 * KEYS * kPieces / 64; load += NW) {
      const int which = load >= KEYS * kPieces / 64 ? 1 : 0, row0 = (load - which * (KEYS * kPieces / 64)) * (64 / kPieces);
      const int key = row0 + lane / kPieces;
      const size_t row = ((size_t)u.b * p.gamma * p.L + own_row(u, first, key)) * p.Hkv + u.hk;
      const uint8_t *src = (const uint8_t *)(which ? p.v_branch : p.k_branch) + (row * kPieces + ((lane % kPieces) ^ swizzle<D>(key))) * 16;
      load_lds16(src, lds_address(which ? v_lds : k_lds) + row0 * D * 2);
    }
    wait_loads();
    __syncthreads();
    f32x16 s[NB];
    tile_scores(s, st, k_lds, kt);
    tile_max<D, NB, TILE_OWN>(s, st, p.scale_log2, first + my_keys, u.own_end, h);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      bf16x8 pf[2];
      tile_probs(pf, s[kb], st, p.scale_log2);
      tile_values(st, pf, v_lds + kb * 32 * D * 2, vt);
    }
    __syncthreads();
  }

  float l = xhalf_sum(st.l), m = st.m;
  if constexpr (KS == 2) {
    // the two halves of the keys: common maximum, then the sum of the accumulators through LDS
    float *buf = (float *)lds + row_wave * (D / 32) * 16 * 64 + lane;
    if (key_wave == 1) {
      if (h == 0) fold_ml[row_wave * 32 + ln][0] = m, fold_ml[row_wave * 32 + ln][1] = l;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) buf[(db * 16 + j) * 64] = st.o[db][j];
    }
    __syncthreads();
    if (key_wave == 1) return;
    const float m1 = fold_ml[row_wave * 32 + ln][0], l1 = fold_ml[row_wave * 32 + ln][1];
    const float m_all = fmaxf(m, m1), base = m_all == -INFINITY ? 0.f : m_all;
    const float f0 = __builtin_amdgcn_exp2f(m - base), f1 = __builtin_amdgcn_exp2f(m1 - base);
    m = m_all, l = l * f0 + l1 * f1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) st.o[db][j] = st.o[db][j] * f0 + buf[(db * 16 + j) * 64] * f1;
  }
  if (r >= u.n_rows) return;
  const float inv = 1.0f / l;
  const size_t grow = out_row(p, u, r);
  if (h == 0) put_sums(p, u, grow, m, l);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      put_out(p, u, grow, db * 32 + q * 8 + h * 4, D,
              f32x4{st.o[db][4 * q], st.o[db][4 * q + 1], st.o[db][4 * q + 2], st.o[db][4 * q + 3]}, inv);
}

// ---------------------------------------------------------------------------------------------------- launch

template <int FMT, int D>
hipError_t launch(const SparseParams &p, hipStream_t stream) {
  const int64_t units = (int64_t)p.B * p.n_groups * p.n_row_tiles * p.Hkv;
  const dim3 grid((unsigned)(units * p.n_split)), block(64 * p.waves);
  const int shape = p.tile_rows * 100 + p.waves;
  if (shape == 1604) {
    hipLaunchKernelGGL((attn_blocks_rows_kernel<FMT, D, 1, 4>), grid, block, 0, stream, p);
  } else if (shape == 3204) {
    hipLaunchKernelGGL((attn_blocks_rows_kernel<FMT, D, 2, 4>), grid, block, 0, stream, p);
  } else if constexpr (D == 256) {
    if (shape != 12804) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_blocks_tile_kernel<FMT, D, 4, 1>), grid, block, 0, stream, p);
  } else {
    switch (shape) {
      case 1608: hipLaunchKernelGGL((attn_blocks_rows_kernel<FMT, D, 1, 8>), grid, block, 0, stream, p); break;
      case 3208: hipLaunchKernelGGL((attn_blocks_rows_kernel<FMT, D, 2, 8>), grid, block, 0, stream, p); break;
      case 6404: hipLaunchKernelGGL((attn_blocks_tile_kernel<FMT, D, 2, 2>), grid, block, 0, stream, p); break;
      case 9606: hipLaunchKernelGGL((attn_blocks_tile_kernel<FMT, D, 3, 2>), grid, block, 0, stream, p); break;
      case 12808: hipLaunchKernelGGL((attn_blocks_tile_kernel<FMT, D, 4, 2>), grid, block, 0, stream, p); break;
      default: return hipErrorInvalidValue;
    }
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
