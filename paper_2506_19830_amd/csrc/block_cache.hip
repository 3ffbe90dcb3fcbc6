// Block cache (gfx950): rows are written into the paged cache in bf16, or quantised in groups of 32 elements that share a
// power of two, and read back.
//
// A group x_0 .. x_31 of a row becomes  code_i = rne(x_i * 2^-E),  E the smallest integer in [-100, 100] with
// max |x_i| <= M * 2^E  (M = 448 for fp8-e4m3, 6 for fp4-e2m1; an all-zero group: -100).  No element saturates unless E is at
// its upper end, the scaling is exact, so the one rounding is the conversion's, and the value 2^E * code_i has at most four
// significant bits: exact in bf16.  Beside the rows every block keeps the smallest and the largest key per channel, of the
// values as stored, in bf16 and therefore without rounding.
#include "la_internal.hpp"

namespace la {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) short i16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

__device__ __forceinline__ float low_bf16(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

template <int CTRL>
__device__ __forceinline__ uint32_t quad_swap(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}

// Eight elements of a row; four neighbouring lanes hold a group.
struct Codes {
  u32x4 w;  // bf16: the elements; fp8: codes in w[0], w[1]; fp4: codes in w[0]
  int e;    // exponent of the group
};

template <int FMT>
__device__ __forceinline__ Codes encode(const u32x4 x) {
  Codes r;
  r.w = x, r.e = 0;
  if constexpr (FMT != FMT_BF16) {
    // magnitudes compare as the numbers that their bits are, two at a time
    u16x2 most = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      const uint32_t w = x[i] & 0x7fff7fffu;
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w));
    }
    uint32_t pair = __builtin_bit_cast(uint32_t, most);
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      const uint32_t other = step == 0 ? quad_swap<0xB1>(pair) : quad_swap<0x4E>(pair);  // lane ^ 1, lane ^ 2
      pair = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, pair), __builtin_bit_cast(u16x2, other)));
    }
    const uint32_t top = max(pair & 0xffffu, pair >> 16);
    // top = m * 2^n with 1 <= m < 2: E = n - 8 for m <= 1.75 (448 = 1.75 * 2^8), n - 2 for m <= 1.5 (6 = 1.5 * 2^2), else one
    // more; subnormal tops come out far below the clamp
    const int n = (int)(top >> 7) - 127;
    const uint32_t frac = top & 0x7fu;
    const int e = FMT == FMT_MX8 ? n - 8 + (frac > 0x60u) : n - 2 + (frac > 0x40u);
    r.e = min(max(e, kExpMin), kExpMax);
    const float scale = pow2(r.e);
    if constexpr (FMT == FMT_MX8) {
      if (e <= kExpMax) {
        i16x2 a = {0, 0}, b = {0, 0};
        const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
        a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(bf16x2, x0), scale, false);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(bf16x2, x1), scale, true);
        b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(bf16x2, x2), scale, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(bf16x2, x3), scale, true);
        r.w[0] = __builtin_bit_cast(uint32_t, a), r.w[1] = __builtin_bit_cast(uint32_t, b);
      } else {   // elements beyond 448 * 2^100 saturate
        float f[8];
        const float inv = pow2(-r.e);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = low_bf16(x[i]) * inv, f[2 * i + 1] = high_bf16(x[i]) * inv;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = fminf(fmaxf(f[i], -448.f), 448.f);
        uint32_t a = 0, b = 0;
        a = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], a, false);
        a = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], a, true);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], b, false);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], b, true);
        r.w[0] = a, r.w[1] = b;
      }
    } else {
      const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
      uint32_t a = 0;  // (the conversion saturates at +-6)
      a = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(a, __builtin_bit_cast(bf16x2, x0), scale, 0);
      a = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(a, __builtin_bit_cast(bf16x2, x1), scale, 1);
      a = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(a, __builtin_bit_cast(bf16x2, x2), scale, 2);
      a = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(a, __builtin_bit_cast(bf16x2, x3), scale, 3);
      r.w[0] = a;
    }
  }
  return r;
}

// The stored values of eight elements, as four bf16 pairs.
template <int FMT>
__device__ __forceinline__ u32x4 decode(const u32x4 w, int e) {
  u32x4 r = w;
  if constexpr (FMT == FMT_MX8) {
    const float s = pow2(e);
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, true));
  } else if constexpr (FMT == FMT_MX4) {
    const float s = pow2(e);
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], s, 3));
  }
  return r;
}

// elem: element offset of the eight elements in the cache
template <int FMT>
__device__ __forceinline__ void put(void *cache, size_t elem, const Codes &c) {
  if constexpr (FMT == FMT_BF16)
    *(u32x4 *)((uint8_t *)cache + elem * 2) = c.w;
  else if constexpr (FMT == FMT_MX8)
    *(u32x2 *)((uint8_t *)cache + elem) = u32x2{c.w[0], c.w[1]};
  else
    *(uint32_t *)((uint8_t *)cache + elem / 2) = c.w[0];
}

template <int FMT>
__device__ __forceinline__ u32x4 get(const void *cache, size_t elem) {
  u32x4 r = {0, 0, 0, 0};
  if constexpr (FMT == FMT_BF16) {
    r = *(const u32x4 *)((const uint8_t *)cache + elem * 2);
  } else if constexpr (FMT == FMT_MX8) {
    const u32x2 t = *(const u32x2 *)((const uint8_t *)cache + elem);
    r[0] = t[0], r[1] = t[1];
  } else {
    r[0] = *(const uint32_t *)((const uint8_t *)cache + elem / 2);
  }
  return r;
}

// Two bf16 values as two signed numbers of the same order, and back.
__device__ __forceinline__ i16x2 ordered(uint32_t w) {
  const i16x2 x = __builtin_bit_cast(i16x2, w);
  return x ^ ((x >> 15) & (short)0x7fff);
}
__device__ __forceinline__ i16x2 ordered(i16x2 x) { return x ^ ((x >> 15) & (short)0x7fff); }

// One workgroup writes the new rows of one (layer, request, block of the cache, KV head): D / 8 threads hold a row, so that
// the bounds of the block come out of the rows while they pass through.  Two rows of K and V to a thread are asked for at once.
// Bound by memory where blocks are filled at once (fp8, 22K tokens of 8 heads of 128: 34 us, 3.9 TB/s), by instructions and
// workgroups that find nothing to do where they have few rows (fp4, blocks of 16, 64 layers x 256 tokens: 26 us, 3.4 TB/s;
// with sizes, bounds and conversions on fp32 values instead of bf16 pairs 28.6).
template <int FMT, int D>
__global__ __launch_bounds__(256) void kv_store_kernel(const BlockStoreParams p) {
  constexpr int kPer = D / 8, kRows = 256 / kPer;
  __shared__ __attribute__((aligned(16))) i16x2 red[2][kRows][D / 2];
  const CommitParams &c = p.c;
  const int b = blockIdx.y, layer = blockIdx.z;
  const int hk = blockIdx.x % c.Hkv, j = blockIdx.x / c.Hkv;
  const int src_g = c.src_branch ? min(max(c.src_branch[b], 0), c.gamma - 1) : 0;
  const int n_own = c.n_own ? min(max(c.n_own[b], 0), c.L) : c.L;
  const int n_chain = c.n_chain ? min(max(c.n_chain[b], 0), c.C) : 0;
  const int P = min(max(c.prefix_lens[b], 0), c.capacity);
  const int n_tok = min(n_chain + n_own, c.capacity - P);
  if (layer == 0 && blockIdx.x == 0 && threadIdx.x == 0) c.new_prefix_lens[b] = P + n_tok;

  const int lb = (P >> c.block_shift) + j;
  const int begin = lb << c.block_shift;
  const int first = max(P, begin), end = min(P + n_tok, begin + c.block_size);
  if (first >= end) return;
  const int blk = c.block_tables ? c.block_tables[(size_t)b * c.max_blocks + lb] : b * c.max_blocks + lb;
  const size_t row0 = ((size_t)blk * c.Hkv + hk) * c.block_size;  // of the block, in rows
  const int d0 = (threadIdx.x % kPer) * 8, r0 = threadIdx.x / kPer;

  i16x2 lo[4], hi[4];   // (bounds are bf16 values: the smallest and the largest as ordered numbers)
#pragma unroll
  for (int i = 0; i < 4; ++i) lo[i] = i16x2{0x7fff, 0x7fff}, hi[i] = i16x2{-0x8000, -0x8000};
  for (int pos0 = first + r0; pos0 < end; pos0 += 2 * kRows) {
    u32x4 kx[2], vx[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int t = min(pos0 + x * kRows, end - 1) - P;
      const bool from_chain = t < n_chain;
      const size_t src = from_chain
                             ? (((size_t)b * c.C + t) * c.Hkv + hk) * D + d0 + (size_t)layer * c.chain_stride
                             : ((((size_t)b * c.gamma + src_g) * c.L + (t - n_chain)) * c.Hkv + hk) * D + d0 +
                                   (size_t)layer * c.branch_stride;
      kx[x] = *(const u32x4 *)((const uint8_t *)(from_chain ? c.k_chain : c.k_branch) + src * 2);
      vx[x] = *(const u32x4 *)((const uint8_t *)(from_chain ? c.v_chain : c.v_branch) + src * 2);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int pos = pos0 + x * kRows;
      if (pos >= end) break;
      const Codes kc = encode<FMT>(kx[x]), vc = encode<FMT>(vx[x]);
      const size_t row = row0 + (pos - begin);
      const size_t dst = row * D + d0 + (size_t)layer * c.cache_stride;
      put<FMT>(c.k_cache, dst, kc);
      put<FMT>(c.v_cache, dst, vc);
      if constexpr (FMT != FMT_BF16) {
        if ((threadIdx.x & 3) == 0) {
          const size_t ge = row * (D / kGroup) + d0 / kGroup + (size_t)layer * p.exp_stride;
          p.k_exp[ge] = (uint8_t)(kc.e + kExpBias);
          p.v_exp[ge] = (uint8_t)(vc.e + kExpBias);
        }
      }
      const u32x4 kv = decode<FMT>(kc.w, kc.e);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = kv[i];
        const i16x2 key = ordered(w);
        lo[i] = __builtin_elementwise_min(lo[i], key), hi[i] = __builtin_elementwise_max(hi[i], key);
      }
    }
  }
  if (!p.k_bounds) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) red[0][r0][d0 / 2 + i] = lo[i], red[1][r0][d0 / 2 + i] = hi[i];
  __syncthreads();
  uint32_t *bounds = (uint32_t *)((__bf16 *)p.k_bounds + ((size_t)blk * c.Hkv + hk) * 2 * D + (size_t)layer * p.bounds_stride);
  const int i = threadIdx.x, which = i / (D / 2), d = i % (D / 2);
  if (i >= D) return;
  const short flip = which ? 0 : -1;   // ~v orders the other way round: the smallest is the largest of the complements
  i16x2 v = red[which][0][d] ^ flip;
#pragma unroll
  for (int r = 1; r < kRows; ++r) v = __builtin_elementwise_max(v, red[which][r][d] ^ flip);
  if (first > begin) v = __builtin_elementwise_max(v, ordered(bounds[i]) ^ flip);  // a block begun earlier
  bounds[i] = __builtin_bit_cast(uint32_t, ordered(v ^ flip));
}

// A thread brings eight elements of a key row and the same of its value row back: 4 to 16 bytes in, 16 or 32 out, neighbouring
// threads next to each other.  Bound by memory (fp4 to bf16, 32K tokens of 8 heads of 128: 35.5 us, 4.8 TB/s).
template <int FMT>
__global__ __launch_bounds__(256) void kv_load_kernel(const BlockLoadParams p) {
  const int b = blockIdx.y, layer = blockIdx.z;
  const int per_row = p.D / 8, per_tok = p.Hkv * per_row;
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int t = (int)(item / per_tok);
  if (t >= p.T) return;
  const int rem = (int)(item - (int64_t)t * per_tok);
  const int hk = rem / per_row, d0 = (rem - hk * per_row) * 8;
  const int64_t pos = (int64_t)(p.first ? p.first[b] : 0) + t;
  if (pos < 0 || pos >= min(p.prefix_lens[b], p.capacity)) return;
  const int lb = (int)(pos >> p.block_shift);
  const int blk = p.block_tables ? p.block_tables[(size_t)b * p.max_blocks + lb] : b * p.max_blocks + lb;
  const size_t row = (((size_t)blk * p.Hkv + hk) << p.block_shift) + (size_t)(pos & ((1 << p.block_shift) - 1));
  const size_t src = row * p.D + d0 + (size_t)layer * p.cache_stride;
  const u32x4 kc = get<FMT>(p.k_cache, src), vc = get<FMT>(p.v_cache, src);
  int ke = 0, ve = 0;
  if constexpr (FMT != FMT_BF16) {
    const size_t ge = row * (p.D / kGroup) + d0 / kGroup + (size_t)layer * p.exp_stride;
    ke = (int)p.k_exp[ge] - kExpBias, ve = (int)p.v_exp[ge] - kExpBias;
  }
  const u32x4 kx = decode<FMT>(kc, ke), vx = decode<FMT>(vc, ve);
  const size_t dst = (((size_t)b * p.T + t) * p.Hkv + hk) * p.D + d0 + (size_t)layer * p.out_stride;
  if (p.out_f32) {
    float *ko = (float *)p.k_out + dst, *vo = (float *)p.v_out + dst;
    *(f32x4 *)ko = f32x4{low_bf16(kx[0]), high_bf16(kx[0]), low_bf16(kx[1]), high_bf16(kx[1])};
    *(f32x4 *)(ko + 4) = f32x4{low_bf16(kx[2]), high_bf16(kx[2]), low_bf16(kx[3]), high_bf16(kx[3])};
    *(f32x4 *)vo = f32x4{low_bf16(vx[0]), high_bf16(vx[0]), low_bf16(vx[1]), high_bf16(vx[1])};
    *(f32x4 *)(vo + 4) = f32x4{low_bf16(vx[2]), high_bf16(vx[2]), low_bf16(vx[3]), high_bf16(vx[3])};
  } else {
    *(u32x4 *)((uint8_t *)p.k_out + dst * 2) = kx;
    *(u32x4 *)((uint8_t *)p.v_out + dst * 2) = vx;
  }
}

template <int FMT>
hipError_t launch_store(const BlockStoreParams &p, hipStream_t stream) {
  const dim3 grid(p.n_dst * p.c.Hkv, p.c.B, p.c.num_layers), block(256);
  switch (p.c.D) {
    case 64: hipLaunchKernelGGL((kv_store_kernel<FMT, 64>), grid, block, 0, stream, p); break;
    case 128: hipLaunchKernelGGL((kv_store_kernel<FMT, 128>), grid, block, 0, stream, p); break;
    case 256: hipLaunchKernelGGL((kv_store_kernel<FMT, 256>), grid, block, 0, stream, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_store(const BlockStoreParams &p, int format, hipStream_t stream) {
  ProfileScope scope(SLOT_KV_STORE, stream);
  switch (format) {
    case FMT_BF16: return launch_store<FMT_BF16>(p, stream);
    case FMT_MX8: return launch_store<FMT_MX8>(p, stream);
    case FMT_MX4: return launch_store<FMT_MX4>(p, stream);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_kv_load(const BlockLoadParams &p, int format, hipStream_t stream) {
  ProfileScope scope(SLOT_KV_LOAD, stream);
  const int64_t items = (int64_t)p.T * p.Hkv * (p.D / 8);
  const dim3 grid((unsigned)((items + 255) / 256), p.B, p.num_layers), block(256);
  switch (format) {
    case FMT_BF16: hipLaunchKernelGGL((kv_load_kernel<FMT_BF16>), grid, block, 0, stream, p); break;
    case FMT_MX8: hipLaunchKernelGGL((kv_load_kernel<FMT_MX8>), grid, block, 0, stream, p); break;
    case FMT_MX4: hipLaunchKernelGGL((kv_load_kernel<FMT_MX4>), grid, block, 0, stream, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace la
