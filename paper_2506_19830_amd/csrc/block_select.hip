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

// 16 bytes per lane from memory to consecutive places in LDS, without registers in between.
__device__ __forceinline__ void load_lds16(const uint8_t *src, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(lds_addr) : "m0");
}
// Until at most N of the wavefront's loads are under way.  (The fences: the compiler does not see the loads' writes to LDS, so
// reads must not be moved over the wait.)
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070 | 0x0F00);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// A wavefront keeps the bounds of 32 blocks (NB tiles of them) in registers as matrix operands while query rows pass, 32 at a
// time.  Groups of at most SLOT rows share such a tile of rows: with rows 8 q .. 8 q + 7 in registers 4 q .. 4 q + 3 of the
// result, the largest of a group's rows is a maximum over registers and the two halves of the wavefront.  Larger groups take
// several tiles (SLOT = 32), which the four wavefronts of a workgroup share in LDS.
//   Everything comes from memory in whole rows and is taken apart in LDS: operands read from memory directly, 16 bytes of 32
// rows per instruction, kept the cache's tag look-ups busy (steps of 320 rows, 2048 blocks: 34 -> 26 us).  A row's 16-byte pieces lie permuted by the row's number, so that the reads of one piece of 16 rows miss no bank.
template <int D, int SLOT, int NB>
__global__ __launch_bounds__(256) void block_score_kernel(const SelectParams p) {
  constexpr int T = D / 16, kShare = 32 / SLOT, kRegs = SLOT / 2;  // groups of a row tile; registers of a group
  constexpr int kPieces = D / 8, kMask = kPieces < 16 ? kPieces - 1 : 15;   // 16-byte pieces of a query row
  // The bounds of 32 blocks, lower and upper ones together or, where nothing else wants the LDS, one after the other: a SIMD
  // then holds four wavefronts instead of two (32 requests of up to 512 blocks: 14.1 -> 13.2 us;
  // 54 groups of 5 rows and 626 blocks: 9.3 -> 7.6).
  constexpr int kHalves = SLOT < 32 ? 1 : 2, kTileBytes = 32 * 2 * D, kBoundBytes = kHalves * kTileBytes;
  constexpr int kRing = 4, kPerWave = kTileBytes / 1024 / 4;        // query tiles in LDS; loads of a wavefront per tile
  __shared__ __attribute__((aligned(16))) uint8_t lds[4 * kBoundBytes];
  static_assert(kRing * kTileBytes <= 4 * kBoundBytes, "the query tiles take the place of the bounds");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane & 31, h = lane >> 5;
  uint32_t id = blockIdx.y + blockIdx.z * 65535u;
  if (id >= (uint32_t)(p.B * p.score_chunks * p.Hkv)) return;
  const int hk = (int)(id % (uint32_t)p.Hkv);
  id /= (uint32_t)p.Hkv;
  const int chunk = (int)(id % (uint32_t)p.score_chunks), b = (int)(id / (uint32_t)p.score_chunks);
  const int tile = (blockIdx.x * 4 + wave) * NB;
  const uint32_t bounds_at = lds_address(lds) + wave * kBoundBytes;
  const int32_t *table = p.block_tables ? p.block_tables + (size_t)b * p.max_blocks : nullptr;
  u32x4 lo[NB][T], hi[NB][T];
  // the table's entries are asked for together with the prefix's length (those behind it are not used); blocks behind the last
  // repeat the last one, or where that is in another tile block 0 of the request
  int blk[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int lb = min((tile + nb) * 32 + ln, p.max_blocks - 1);
    blk[nb] = table ? table[lb] : b * p.max_blocks + lb;
  }
  const int n = prefix_blocks(p, b);
  if (n <= p.max_sel || blockIdx.x * 4 * NB * 32 >= (uint32_t)n) return;  // all blocks are taken / no such blocks
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int last = n - 1 - (tile + nb) * 32;   // of the tile's blocks; negative: no such tile, which then repeats block 0
    if (last < 0) blk[nb] = table ? table[0] : b * p.max_blocks;
    const int edge = __shfl(blk[nb], min(max(last, 0), 31));
    if (ln > last) blk[nb] = edge;
  }
  const int per_req = p.gamma * p.n_groups;
  const int first = chunk * p.score_groups, end = min(first + p.score_groups, per_req);
  // rows of a group, and the place of its row r
  auto rows_of = [&](int group, int &n_rows) __attribute__((always_inline)) {
    const int g = group / p.n_groups, t0 = (group - g * p.n_groups) * p.group_len;
    n_rows = min(p.group_len, p.L - t0) * p.G;
    return (const uint8_t *)p.q + ((((size_t)b * p.gamma + g) * p.L + t0) * p.Hq + hk * p.G) * D * 2;
  };
  auto place = [&](int r) __attribute__((always_inline)) { return ((size_t)(r / p.G) * p.Hq + r % p.G) * D * 2; };
  u32x4 q[T];   // (SLOT < 32: the rows of the next groups, under way)
  auto request_rows = [&](int group) __attribute__((always_inline)) {
    int n_rows;
    const uint8_t *qs = rows_of(min(group + ln / SLOT, end - 1), n_rows);
    qs += place(min(ln % SLOT, n_rows - 1)) + h * 16;
#pragma unroll
    for (int t = 0; t < T; ++t) q[t] = *(const u32x4 *)(qs + t * 32);
  };
  auto request_bounds = [&](int nb, int upper) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kTileBytes / 1024; ++i) {
      const int x = i * (64 / kPieces) + lane / kPieces;           // the block among the 32
      const int from = __shfl(blk[nb], x);
      const int piece = (lane % kPieces) ^ (x & kMask);
      load_lds16((const uint8_t *)p.k_bounds + ((((size_t)from * p.Hkv + hk) * 2 + upper) * kPieces + piece) * 16,
                 bounds_at + upper % kHalves * kTileBytes + i * 1024);
    }
  };
  auto take_bounds = [&](u32x4 (&x)[T], int upper) __attribute__((always_inline)) {
    const uint8_t *mine = lds + wave * kBoundBytes + upper % kHalves * kTileBytes + ln * 2 * D;
#pragma unroll
    for (int t = 0; t < T; ++t) x[t] = *(const u32x4 *)(mine + (((2 * t + h) ^ (ln & kMask)) << 4));
  };
  // (what comes next to the same place waits until this is in registers)
  auto wait_taken = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    request_bounds(nb, 0);
    if (kHalves == 2) request_bounds(nb, 1);
    if (SLOT < 32 && nb == 0) request_rows(first);
    wait_loads<0>();
    take_bounds(lo[nb], 0);
    if (kHalves == 1) {
      wait_taken();
      request_bounds(nb, 1);
      wait_loads<0>();
    }
    take_bounds(hi[nb], 1);
    wait_taken();
  }
  auto tile_scores = [&](const u32x4 (&q)[T], f32x16 (&s)[NB]) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 16; ++j) s[nb][j] = 0.f;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      u32x4 neg, pos;
      split_signs(q[t], neg, pos);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, neg), __builtin_bit_cast(bf16x8, lo[nb][t]), s[nb], 0, 0, 0);
        s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, pos), __builtin_bit_cast(bf16x8, hi[nb][t]), s[nb], 0, 0, 0);
      }
    }
  };
  auto store = [&](int group, int nb, float best) __attribute__((always_inline)) {
    const int lb = (tile + nb) * 32 + ln;
    if (h == 0 && lb < n) p.score[(((size_t)b * per_req + group) * p.Hkv + hk) * p.n_max + lb] = best;
  };
  if constexpr (SLOT == 32) {
    const int per_group = (p.group_len * p.G + 31) / 32, total = (end - first) * per_group;
    int next_group = first, next_part = 0;   // of the tile that is requested next
    auto request = [&](int slot) __attribute__((always_inline)) {
      int n_rows;
      const uint8_t *base = rows_of(next_group, n_rows);
#pragma unroll
      for (int j = 0; j < kPerWave; ++j) {
        const int row = ((wave * kPerWave + j) * 64 + lane) / kPieces, r = min(next_part * 32 + row, n_rows - 1);  // (surplus rows repeat the last one)
        load_lds16(base + place(r) + (((lane % kPieces) ^ (row & kMask)) << 4), lds_address(lds) + slot * kTileBytes + (wave * kPerWave + j) * 1024);
      }
      if (++next_part == per_group) next_part = 0, next_group = min(next_group + 1, end - 1);  // (behind the last tile: others again)
    };
    __syncthreads();   // every wavefront has its bounds in registers
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) request(i);
    float best[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) best[nb] = -INFINITY;
    int group = first, part = 0;
    for (int i = 0; i < total; ++i) {
      wait_loads<(kRing - 2) * kPerWave>();
      __syncthreads();   // tile i is there, and tile i - 1 has been read by all
      request((i + kRing - 1) & (kRing - 1));
      const uint8_t *mine = lds + (i & (kRing - 1)) * kTileBytes + ln * 2 * D;
#pragma unroll
      for (int t = 0; t < T; ++t) q[t] = *(const u32x4 *)(mine + (((2 * t + h) ^ (ln & kMask)) << 4));
      f32x16 s[NB];
      tile_scores(q, s);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 16; ++j) best[nb] = fmaxf(best[nb], s[nb][j]);
      if (++part == per_group) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          store(group, nb, xhalf_max(best[nb]));
          best[nb] = -INFINITY;
        }
        ++group, part = 0;
      }
    }
    wait_loads<0>();
  } else {
    for (int group = first; group < end; group += kShare) {
      f32x16 s[NB];
      tile_scores(q, s);
      if (group + kShare < end) request_rows(group + kShare);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int q = 0; q < kShare; ++q) {
          float best = s[nb][q * kRegs];
#pragma unroll
          for (int j = 1; j < kRegs; ++j) best = fmaxf(best, s[nb][q * kRegs + j]);
          best = xhalf_max(best);
          if (group + q < end) store(group + q, nb, best);
        }
    }
  }
  if (chunk == 0 && tile * 32 < n) {  // the largest magnitude among the tiles' bounds, once per request and head
    uint32_t top = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a = lo[nb][t][i], z = hi[nb][t][i];
          top = max(top, max(max(a << 16 & 0x7fffffffu, a & 0x7fff0000u), max(z << 16 & 0x7fffffffu, z & 0x7fff0000u)));
        }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
    if (lane == 0) p.top[((size_t)b * p.Hkv + hk) * p.n_tiles + tile / NB] = __builtin_bit_cast(float, top);
  }
}

constexpr int kListed = 1024;  // blocks in doubt that are held in LDS
constexpr int kPairs = 1024;   // (block, row) pairs whose exact sums decide them

// LDS of a workgroup of NT threads that picks blocks.  The functions on it are called by all of its threads.
template <int NT>
struct Shared {
  uint32_t hist[256];
  uint32_t key_lo[NT / 64], key_hi[NT / 64];
  float size_q[NT / 64], size_k[NT / 64];
  uint32_t bin, bin_above, bin_count, n_list, n_doubt, n_sure;
  uint32_t list[64];
  int doubt[kListed];
  unsigned long long doubt_key[kListed];
  uint8_t doubt_taken[kListed];
  uint32_t n_pairs, pair_row[kPairs];   // (a group may have up to 2^30 rows)
  uint16_t pair_doubt[kPairs];          // index into doubt
  int count[8 * (NT / 64)];
};

// The bin (counted from the top) of sh.hist in which item `rank` from the top lies: sh.bin, the items above it and in it.
template <int NT>
__device__ __forceinline__ void find_bin(Shared<NT> &sh, uint32_t rank) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t own = 0, incl = 0;
  if (wave < 4) {
    own = incl = sh.hist[255 - tid];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t up = (uint32_t)__shfl_up((int)incl, off);
      if (lane >= off) incl += up;
    }
    if (lane == 63) sh.key_lo[wave] = incl;
  }
  __syncthreads();
  if (wave < 4) {
    for (int w = 0; w < wave; ++w) incl += sh.key_lo[w];
    if (incl >= rank && incl - own < rank) sh.bin = 255 - tid, sh.bin_above = incl - own, sh.bin_count = own;
  }
  __syncthreads();
}

// Item `rank` from the top among the keys (0: not an item) that `for_each` visits, and how many items lie above it: eight
// bits at a time, from any number of items.
template <int NT, typename Key, typename F>
__device__ Key key_of_rank(Shared<NT> &sh, uint32_t rank, F for_each, uint32_t *above) {
  constexpr int kBits = (int)sizeof(Key) * 8;
  Key prefix = 0;
  uint32_t left = rank;
  for (int shift = kBits - 8; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.bin = sh.bin_above = 0;
    __syncthreads();
    for_each([&](Key k) {
      if (k != 0 && (shift + 8 >= kBits || (k >> (shift + 8)) == (prefix >> (shift + 8))))
        atomicAdd(&sh.hist[(uint32_t)(k >> shift) & 255u], 1u);
    });
    __syncthreads();
    find_bin(sh, left);
    prefix |= (Key)sh.bin << shift;
    left -= sh.bin_above;
    __syncthreads();
  }
  *above = rank - left;
  return prefix;
}

// One workgroup picks the blocks of one group and KV head from their scores.  Up to 8 NT candidates stay in registers (IN_REG).
// Bound by the latency of a dozen dependent steps over a few hundred numbers (256 groups, up to 512 candidates: 9.8 us), and with
// many rows by the second look at the blocks in doubt (64 groups of 320 rows, 2048 candidates: 20.8 us).
template <int D, int NT, bool IN_REG>
__global__ __launch_bounds__(NT) void block_pick_kernel(const SelectParams p) {
  constexpr int kItems = 8, kWaves = NT / 64;
  __shared__ Shared<NT> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t id = blockIdx.x;
  const size_t unit = id;
  const int hk = (int)(id % (uint32_t)p.Hkv);
  id /= (uint32_t)p.Hkv;
  const int per_req = p.gamma * p.n_groups;
  const int b = (int)(id / (uint32_t)per_req), group = (int)(id % (uint32_t)per_req);
  int32_t *out = p.blocks + unit * p.max_sel;
  const float *score = p.score + unit * p.n_max;
  const int c0 = p.keep_first;   // the first candidate
  float item[kItems];
  if (IN_REG && p.n_max > p.max_sel) {   // (asked for together with the prefix's length; there are n_max places)
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = c0 + tid + k * NT;
      item[k] = i < p.n_max ? score[i] : 0.f;
    }
  }
  // the largest sum of magnitudes of a row and the largest magnitude of a bound give the error of the scores
  const int g = group / p.n_groups, t0 = (group - g * p.n_groups) * p.group_len;
  const int n_rows = min(p.group_len, p.L - t0) * p.G;
  const size_t tok0 = ((size_t)b * p.gamma + g) * p.L + t0;
  auto row_of = [&](int r) __attribute__((always_inline)) {
    return (const uint8_t *)p.q + ((tok0 + r / p.G) * p.Hq + hk * p.G + r % p.G) * D * 2;
  };
  float size_q = 0.f, size_k = 0.f;
  constexpr int kPer = D / 8;  // lanes that share a row
  for (int r0 = 0; r0 < n_rows && p.n_max > p.max_sel; r0 += NT / kPer) {
    const int r = r0 + tid / kPer;
    float a = 0.f;
    if (r < n_rows) {
      const u32x4 x = *(const u32x4 *)(row_of(r) + (tid % kPer) * 16);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        a += __builtin_bit_cast(float, x[w] << 16 & 0x7fffffffu) + __builtin_bit_cast(float, x[w] & 0x7fff0000u);
    }
#pragma unroll
    for (int off = 1; off < kPer; off <<= 1) a += __shfl_xor(a, off);
    size_q = fmaxf(size_q, a);
  }
  const int n = prefix_blocks(p, b);
  if (n <= p.max_sel) {
    for (int i = tid; i < p.max_sel; i += NT) out[i] = i < n ? i : -1;
    if (tid == 0) p.count[unit] = n;
    return;
  }
  const int c1 = n - p.keep_last;                              // candidates c0 .. c1 - 1
  const int want = p.max_sel - p.keep_first - p.keep_last;     // fewer than there are
  if (tid == 0) p.count[unit] = p.max_sel;
  for (int i = tid; i < c0; i += NT) out[i] = i;
  for (int i = tid; i < p.keep_last; i += NT) out[c0 + want + i] = c1 + i;
  if (want == 0) return;
  // f(place of the candidate, its score, its number among the thread's)
  auto for_each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (IN_REG) {
#pragma unroll
      for (int k = 0; k < kItems; ++k)
        if (c0 + tid + k * NT < c1) f(c0 + tid + k * NT, item[k], k);
    } else {
      for (int i = c0 + tid; i < c1; i += NT) f(i, score[i], 0);
    }
  };

  for (int i = tid; i * p.top_blocks < n; i += NT) size_k = fmaxf(size_k, p.top[((size_t)b * p.Hkv + hk) * p.n_tiles + i]);
  uint32_t key_lo = 0xffffffffu, key_hi = 0;   // the smallest and the largest key
  for_each([&](int, float s, int) { key_lo = min(key_lo, order_key(s)), key_hi = max(key_hi, order_key(s)); });
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    size_q = fmaxf(size_q, __shfl_xor(size_q, off)), size_k = fmaxf(size_k, __shfl_xor(size_k, off));
    key_lo = min(key_lo, (uint32_t)__shfl_xor((int)key_lo, off)), key_hi = max(key_hi, (uint32_t)__shfl_xor((int)key_hi, off));
  }
  if (lane == 0) sh.size_q[wave] = size_q, sh.size_k[wave] = size_k, sh.key_lo[wave] = key_lo, sh.key_hi[wave] = key_hi;
  if (tid == 0) sh.n_list = sh.n_doubt = sh.n_sure = sh.n_pairs = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    size_q = fmaxf(size_q, sh.size_q[w]), size_k = fmaxf(size_k, sh.size_k[w]);
    key_lo = min(key_lo, sh.key_lo[w]), key_hi = max(key_hi, sh.key_hi[w]);
  }
  const float err = kScoreError<D> * 1.01f * size_q * size_k + 1e-30f;
  // where a sum may have left fp32 the rounded scores say nothing: every block is in doubt  (size_q: its own sum may have, too)
  const bool lost = size_q * size_k > 0x1p126f || size_q > 0x1p126f;

  // t, the score of rank `want`: bins of equal width between the smallest and the largest key, then inside the bin it lies in,
  // until a wavefront can hold that
  uint32_t left = (uint32_t)want;
  while (key_lo != key_hi) {
    const int shift = max(0, 24 - (int)__builtin_clz(key_hi - key_lo));
    __syncthreads();
    if (tid < 256) sh.hist[tid] = 0;
    if (tid == 0) sh.bin = sh.bin_above = sh.bin_count = 0;
    __syncthreads();
    for_each([&](int, float s, int) {
      const uint32_t k = order_key(s);
      if (k >= key_lo && k <= key_hi) atomicAdd(&sh.hist[(k - key_lo) >> shift], 1u);
    });
    __syncthreads();
    find_bin(sh, left);
    left -= sh.bin_above;
    const uint32_t count = sh.bin_count;
    key_lo += sh.bin << shift;
    key_hi = min(key_hi, key_lo + ((1u << shift) - 1u));
    if (key_lo == key_hi || count > 64) continue;
    for_each([&](int, float s, int) {
      const uint32_t k = order_key(s);
      if (k >= key_lo && k <= key_hi) sh.list[atomicAdd(&sh.n_list, 1u) & 63u] = k;
    });
    __syncthreads();
    const uint32_t mine = lane < (int)count ? sh.list[lane] : 0u;
    uint32_t above = 0, same = 0;
    for (uint32_t j = 0; j < count; ++j) {
      const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)mine, (int)j);
      above += k > mine ? 1u : 0u, same += k == mine ? 1u : 0u;
    }
    const uint64_t hit = __builtin_amdgcn_ballot_w64(lane < (int)count && above < left && left <= above + same);
    key_lo = key_hi = (uint32_t)__builtin_amdgcn_readlane((int)mine, hit ? __builtin_ctzll(hit) : 0);
  }
  const float t = key_value(key_lo);
  const float sure = t + 2.f * err, out_of = t - 2.f * err;  // above: certainly taken; below: certainly not
  auto taken = [&](float s) __attribute__((always_inline)) { return s > sure && !lost; };
  auto in_doubt = [&](float s) __attribute__((always_inline)) { return (s >= out_of && !(s > sure)) || lost; };

  int slot[kItems];
  for_each([&](int i, float s, int k) {
    if (taken(s)) {
      atomicAdd(&sh.n_sure, 1u);
    } else if (in_doubt(s)) {
      const uint32_t at = atomicAdd(&sh.n_doubt, 1u);
      if (at < kListed) sh.doubt[at] = i, sh.doubt_key[at] = 0;
      if constexpr (IN_REG) slot[k] = (int)at;
    }
  });
  __syncthreads();
  const uint32_t n_doubt = sh.n_doubt, need = (uint32_t)want - sh.n_sure;
  const bool listed = IN_REG && n_doubt <= kListed;

  auto bounds_of = [&](int lb) __attribute__((always_inline)) {
    const int blk = p.block_tables ? p.block_tables[(size_t)b * p.max_blocks + lb] : b * p.max_blocks + lb;
    return (const uint8_t *)p.k_bounds + ((size_t)blk * p.Hkv + hk) * 4 * D;
  };
  // The exact sum of row r and block lb, eight lanes to a row.
  auto exact_row = [&](int lb, int r) __attribute__((always_inline)) {
    const uint8_t *bs = bounds_of(lb), *qs = row_of(r);
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const int at = (c * 8 + (lane & 7)) * 16;
      const u32x4 q = *(const u32x4 *)(qs + at), lo = *(const u32x4 *)(bs + at), hi = *(const u32x4 *)(bs + 2 * D + at);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t a = (q[w] << 16) >> 31 ? lo[w] << 16 : hi[w] << 16;
        const uint32_t z = q[w] >> 31 ? lo[w] & 0xffff0000u : hi[w] & 0xffff0000u;
        sum += (double)__builtin_bit_cast(float, q[w] << 16) * (double)__builtin_bit_cast(float, a);
        sum += (double)__builtin_bit_cast(float, q[w] & 0xffff0000u) * (double)__builtin_bit_cast(float, z);
      }
    }
    sum += __shfl_xor(sum, 1), sum += __shfl_xor(sum, 2);
    return sum + __shfl_xor(sum, 4);
  };
  // One wavefront: the largest over rows r0 .. r0 + 7.
  auto exact_rows = [&](int lb, int r0) __attribute__((always_inline)) {
    double s = exact_row(lb, min(r0 + (lane >> 3), n_rows - 1));
    s = fmax(s, __shfl_xor(s, 8)), s = fmax(s, __shfl_xor(s, 16));
    return fmax(s, __shfl_xor(s, 32));
  };

  if (listed) {
    bool all_rows = true;
    if (n_doubt > need && n_rows > 8) {
      // of a group's rows only those can hold a block's largest exact sum whose rounded sum is within 2 e of the largest
      // rounded one: the sums of the blocks in doubt once more, 32 of them at a time, and the few rows listed
      for (int k0 = 0; k0 < (int)n_doubt; k0 += 32) {
        const int k = k0 + (lane & 31), h = lane >> 5, lb = sh.doubt[min(k, (int)n_doubt - 1)];
        const uint8_t *bs = bounds_of(lb) + h * 16;
        const float least = score[lb] - 2.f * err;
        for (int r0 = wave * 32; r0 < n_rows; r0 += kWaves * 32) {
          const uint8_t *qs = row_of(min(r0 + (lane & 31), n_rows - 1)) + h * 16;
          f32x16 s;
#pragma unroll
          for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
          for (int t = 0; t < D / 16; ++t) {
            u32x4 neg, pos;
            split_signs(*(const u32x4 *)(qs + t * 32), neg, pos);
            const bf16x8 lo = *(const bf16x8 *)(bs + t * 32), hi = *(const bf16x8 *)(bs + 2 * D + t * 32);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, neg), lo, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, pos), hi, s, 0, 0, 0);
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int r = r0 + (j >> 2) * 8 + h * 4 + (j & 3);
            // (nothing is counted once there are too many: the pairs of many rows and blocks would pass 32 bits)
            if (k < (int)n_doubt && r < n_rows && (s[j] >= least || lost) &&
                __hip_atomic_load(&sh.n_pairs, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) <= kPairs) {
              const uint32_t at = atomicAdd(&sh.n_pairs, 1u);
              if (at < kPairs) sh.pair_row[at] = (uint32_t)r, sh.pair_doubt[at] = (uint16_t)k;
            }
          }
        }
      }
      __syncthreads();
      const int n_pairs = (int)sh.n_pairs;
      all_rows = n_pairs > kPairs;
      for (int i0 = wave * 8; i0 < n_pairs && !all_rows; i0 += kWaves * 8) {
        const int pair = min(i0 + (lane >> 3), n_pairs - 1), k = sh.pair_doubt[pair];
        const double s = exact_row(sh.doubt[k], (int)sh.pair_row[pair]);
        if ((lane & 7) == 0) atomicMax(&sh.doubt_key[k], (unsigned long long)order_key64(s));
      }
    }
    if (n_doubt > need) {
      // (block, part of the rows) in turn, kWaves of them a step; their number may pass 32 bits
      const int parts = (n_rows + 7) / 8, next_k = kWaves / parts, next_part = kWaves % parts;
      int k = wave / parts, part = wave % parts;
      while (all_rows && k < (int)n_doubt) {
        const double s = exact_rows(sh.doubt[k], part * 8);
        if (lane == 0) atomicMax(&sh.doubt_key[k], (unsigned long long)order_key64(s));
        k += next_k, part += next_part;
        if (part >= parts) part -= parts, ++k;
      }
      __syncthreads();
    }
    for (int k = tid; k < (int)n_doubt; k += NT) {
      uint32_t better = 0;
      if (n_doubt > need) {
        const unsigned long long mine = sh.doubt_key[k];
        const int mine_i = sh.doubt[k];
        for (uint32_t j = 0; j < n_doubt; ++j) {
          const unsigned long long other = sh.doubt_key[j];
          better += other > mine || (other == mine && sh.doubt[j] < mine_i) ? 1u : 0u;
        }
      }
      sh.doubt_taken[k] = better < need ? 1 : 0;
    }
    __syncthreads();
    // the list, in ascending order: how many each wavefront takes of each of its eight rows of candidates, then their places
    uint32_t takes = 0;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      bool take = false;
      if (c0 + tid + k * NT < c1) take = taken(item[k]) || (in_doubt(item[k]) && sh.doubt_taken[slot[k]]);
      const uint64_t mask = __builtin_amdgcn_ballot_w64(take);
      if (lane == 0) sh.count[k * kWaves + wave] = __popcll(mask);
      takes |= (uint32_t)take << k;
    }
    __syncthreads();
    constexpr int kCounts = kItems * kWaves, kPerLane = (kCounts + 63) / 64;
    int own[kPerLane], sum = 0;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
      own[j] = lane * kPerLane + j < kCounts ? sh.count[lane * kPerLane + j] : 0;
      sum += own[j];
    }
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int up = __shfl_up(incl, off);
      if (lane >= off) incl += up;
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int at = k * kWaves + wave, holder = at / kPerLane;  // of the counts of row k and this wavefront
      int before = __builtin_amdgcn_readlane(incl - sum, holder);
#pragma unroll
      for (int j = 0; j + 1 < kPerLane; ++j)
        if (j < at % kPerLane) before += __builtin_amdgcn_readlane(own[j], holder);
      const bool take = (takes >> k) & 1;
      const int place = before + __popcll(__builtin_amdgcn_ballot_w64(take) & ((1ull << lane) - 1));
      if (take && place < want) out[c0 + place] = c0 + tid + k * NT;
    }
    return;
  }

  // Any number of candidates and of blocks in doubt: exact scores and all decisions go through memory.
  double *exact = p.exact + unit * p.n_max;
  unsigned long long exact_t = 0;
  uint32_t ties = n_doubt;  // blocks at the threshold that are taken, the lowest indices first
  if (n_doubt > need) {
    for (int i0 = c0; i0 < c1; i0 += NT) {
      const int i = i0 + tid;
      __syncthreads();
      if (tid == 0) sh.n_doubt = 0;
      __syncthreads();
      if (i < c1 && in_doubt(score[i])) sh.doubt[atomicAdd(&sh.n_doubt, 1u) % kListed] = i;  // (at most NT <= kListed)
      __syncthreads();
      for (int k = wave; k < (int)sh.n_doubt; k += kWaves) {
        double s = -INFINITY;
        for (int r0 = 0; r0 < n_rows; r0 += 8) s = fmax(s, exact_rows(sh.doubt[k], r0));
        if (lane == 0) exact[sh.doubt[k]] = s;
      }
    }
    __syncthreads();
    uint32_t exact_above;
    exact_t = key_of_rank<NT, unsigned long long>(
        sh, need,
        [&](auto visit) {
          for (int i = c0 + tid; i < c1; i += NT) visit(in_doubt(score[i]) ? (unsigned long long)order_key64(exact[i]) : 0ull);
        },
        &exact_above);
    ties = need - exact_above;
  }
  int at = 0;
  uint32_t tied = 0;
  for (int i0 = c0; i0 < c1; i0 += NT) {
    const int i = i0 + tid;
    bool take = false, tie = false;
    if (i < c1) {
      const float s = score[i];
      take = taken(s);
      if (!take && in_doubt(s)) {
        if (n_doubt > need) {
          const unsigned long long k = order_key64(exact[i]);
          take = k > exact_t, tie = k == exact_t;
        } else {
          take = true;
        }
      }
    }
    const uint64_t tie_mask = __builtin_amdgcn_ballot_w64(tie), below = (1ull << lane) - 1;
    __syncthreads();
    if (lane == 0) sh.count[wave] = __popcll(tie_mask);
    __syncthreads();
    uint32_t rank = tied + (uint32_t)__popcll(tie_mask & below);
    for (int w = 0; w < kWaves; ++w) rank += w < wave ? (uint32_t)sh.count[w] : 0u, tied += (uint32_t)sh.count[w];
    take |= tie && rank < ties;
    const uint64_t mask = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) sh.count[kWaves + wave] = __popcll(mask);
    __syncthreads();
    int place = at + __popcll(mask & below);
    for (int w = 0; w < kWaves; ++w) place += w < wave ? sh.count[kWaves + w] : 0, at += sh.count[kWaves + w];
    if (take && place < want) out[c0 + place] = i;
  }
}

template <int D, int SLOT, int NB>
hipError_t launch_score(SelectParams &p, hipStream_t stream) {
  ProfileScope scope(SLOT_BLOCK_SCORE, stream);
  const int64_t groups = (int64_t)p.gamma * p.n_groups;
  const int64_t row_tiles = (groups + 32 / SLOT - 1) / (32 / SLOT);
  p.top_blocks = 32 * NB;
  const int64_t tiles = (p.n_max + 32 * NB - 1) / (32 * NB), wgs = (tiles + 3) / 4;
  // wavefronts that go through several groups read their blocks' bounds once: as many as fill the chip about four times over
  // (2048 workgroups), the groups shared out among them
  int64_t chunks = (2048 + wgs * p.B * p.Hkv - 1) / (wgs * p.B * p.Hkv);
  chunks = chunks < row_tiles ? chunks : row_tiles;
  const int64_t share = (row_tiles + chunks - 1) / chunks;
  chunks = (row_tiles + share - 1) / share;
  p.score_chunks = (int)chunks;
  p.score_groups = (int)(share * (32 / SLOT));
  const int64_t units = chunks * p.B * p.Hkv;
  const dim3 grid((unsigned)wgs, (unsigned)(units < 65535 ? units : 65535), (unsigned)((units + 65534) / 65535));
  hipLaunchKernelGGL((block_score_kernel<D, SLOT, NB>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch(SelectParams p, hipStream_t stream) {
  const int rows = p.group_len * p.G;
  if (p.n_max > p.max_sel) {
    hipError_t e;
    if (rows <= 8)
      e = launch_score<D, 8, 1>(p, stream);
    else if (rows <= 16)
      e = launch_score<D, 16, 1>(p, stream);
    else
      e = launch_score<D, 32, D <= 128 ? 2 : 1>(p, stream);
    if (e != hipSuccess) return e;
  }
  ProfileScope scope(SLOT_BLOCK_PICK, stream);
  const dim3 grid((unsigned)((int64_t)p.B * p.gamma * p.n_groups * p.Hkv));
  if (p.n_max > 8 * 1024)
    hipLaunchKernelGGL((block_pick_kernel<D, 1024, false>), grid, dim3(1024), 0, stream, p);
  else if (block_pick_threads(p.n_max, rows) == 1024)
    hipLaunchKernelGGL((block_pick_kernel<D, 1024, true>), grid, dim3(1024), 0, stream, p);
  else
    hipLaunchKernelGGL((block_pick_kernel<D, 256, true>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

// Sixteen wavefronts where one group's work can use them: more candidates than four hold, or exact scores over many rows.
int block_pick_threads(int n_max, int rows) { return n_max > 8 * 256 || rows > 64 ? 1024 : 256; }

hipError_t launch_block_select(const SelectParams &p, hipStream_t stream) {
  switch (p.D) {
    case 64: return launch<64>(p, stream);
    case 128: return launch<128>(p, stream);
    case 256: return launch<256>(p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace la
