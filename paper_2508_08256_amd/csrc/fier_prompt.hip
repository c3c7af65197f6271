// Causal attention of many new tokens per sequence: whole prompts packed one after the other (fier_prefill_attn), and
// chunks over the rows of a cache (fier_chunk_attn).
//   Token i of a sequence's n attends over the rows 0 .. first + i; first = 0 for prompts, the length before the chunk for a
// cache.  A unit (sequence, kv head) has n * n_rep query rows, row = token * n_rep + head of the group, so that the heads that
// share K and V share their tiles too.
#include <float.h>

#include "fier.h"
#include "fier_dev.h"
#include "fier_kernels.h"

namespace fier {

typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx2_t __attribute__((ext_vector_type(2)));

constexpr int kTile = 64;      // rows of K and V per step
constexpr int kRowBytes = 2 * kD;
constexpr float kLargeScaled = 0x1p22f;  // scaled logits from here on are rounded before the maximum is subtracted

template <int DT>
__device__ __forceinline__ floatx16_t mfma_32x32x16(const uint4& a, const uint4& b, floatx16_t c) {
  if (DT == DT_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// two floats rounded to nearest even
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const floatx2_t x = {a, b};
  if (DT == DT_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, half2_t));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
}

__device__ __forceinline__ float halves_max(float x) {
  typedef unsigned int u2_t __attribute__((ext_vector_type(2)));
  const u2_t a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  typedef unsigned int u2_t __attribute__((ext_vector_type(2)));
  const u2_t a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// a * b rounded by itself, never the inside of a fused multiply-add
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

typedef __attribute__((address_space(3))) char lds_char;
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 lds_read16(const lds_char* p) {
  const u32x4_t v = *(const __attribute__((address_space(3))) u32x4_t*)p;
  return make_uint4(v.x, v.y, v.z, v.w);
}
// Four 2-byte columns of four rows per lane: of the 16 lanes' addresses, those of lanes 4 r .. 4 r + 3 are row r, and lane i
// receives column i of rows 0..3.
__device__ __forceinline__ uint2 lds_read_transposed(const lds_char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)p));
}

// Where a unit's K / V rows lie: a cache, or packed prompts with strides (bytes) between tokens.
struct TileRows {
  const char *k, *v;  // the tile's first row
};
__device__ __forceinline__ TileRows tile_rows(const PromptArgs& a, int unit, int head, int lo, int t0) {
  if (a.from_cache) {
    const size_t off = a.lay.rows_of(unit).row(t0) * kRowBytes;
    return {a.k + off, a.v + off};
  }
  return {a.k + (size_t)(lo + t0) * a.k_stride + head * kRowBytes, a.v + (size_t)(lo + t0) * a.v_stride + head * kRowBytes};
}

// 64 rows into LDS by NW wavefronts, 4 rows (1 KiB) per load.  The 16-byte chunks of a row are permuted so that the reads of
// both products meet no bank twice: K chunk c at c ^ (row & 15); V's pairs of chunks p at p ^ (row & 3) << 1 ^ (row >> 2 & 1).
template <int NW, bool V>
__device__ __forceinline__ void load_tile(const char* src, int64_t stride, int rows, lds_char* dst, int wave, int lane) {
#pragma unroll
  for (int j = 0; j < kTile / 4 / NW; ++j) {
    const int first = 4 * (j * NW + wave);
    const int row = first + (lane >> 4);
    const int c = lane & 15;
    const int chunk = V ? c ^ (((row & 3) << 2) | ((row >> 1) & 2)) : c ^ (row & 15);
    const char* p = src + (int64_t)(row < rows ? row : rows - 1) * stride + chunk * 16;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)(dst + first * kRowBytes), 16, 0, 0);
  }
}

// Query rows 32 wave .. + 31 of the workgroup's 128 per wavefront; K and V tiles of 64 rows shared through LDS.
//   S^T = K Q^T (rows = tokens, columns = query rows): lane (n, h) holds the logits of its query row n for the tokens
// 8 i + 4 h + 0..3 of every 32, which is the B operand of O^T += V^T P^T as it stands, the tokens of a product of 16 taken in
// the order 4 h, 8 + 4 h.  V^T comes out of LDS by transposing reads.  Nothing crosses lanes but the maximum over the halves.
template <int DT>
__global__ __launch_bounds__(256) void prompt_attn_kernel(PromptArgs a) {
  __shared__ __attribute__((aligned(16))) char tiles[2 * kTile * kRowBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int unit = (int)(blockIdx.x % (unsigned)a.units), tile_row = (int)(blockIdx.x / (unsigned)a.units);
  const int b = unit / a.n_kv_heads, head = unit - b * a.n_kv_heads;
  const PromptSpan sp = a.span(b);
  const int row0 = (a.row_tiles - 1 - tile_row) * 128;  // the longest rows first
  const int n_rows = sp.n * a.n_rep;
  if (row0 >= n_rows) return;
  const int last = (row0 + 127 < n_rows ? row0 + 127 : n_rows - 1) / a.n_rep;
  const int n_kv = min(sp.first + last + 1, a.kv_cap);
  int row = row0 + wave * 32 + n;
  const bool there = row < n_rows;
  row = there ? row : n_rows - 1;
  const int tok = row / a.n_rep, qh = head * a.n_rep + row - tok * a.n_rep;
  const int lim = min(sp.first + tok + 1, a.kv_cap);
  const char* qp = a.q + (size_t)(sp.lo + tok) * a.q_stride + qh * kRowBytes;
  uint4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = a.load_q(qp + s * 32 + h * 16);
  lds_char* const kt = (lds_char*)tiles;
  lds_char* const vt = kt + kTile * kRowBytes;
  const lds_char* const kr = kt + n * kRowBytes;
  const int r4 = (lane & 15) >> 2, g1 = (lane >> 4) & 1;
  const lds_char* const vr = vt + (4 * h + r4) * kRowBytes + (lane & 3) * 8;
  floatx16_t o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = floatx16_t{0.f};
  float m = -FLT_MAX, l = 0.f;
  bool large = false;
  constexpr float kBias = DT == DT_F16 ? 7.f : 0.f;
  const float c = a.scale;
  for (int t0 = 0; t0 < n_kv; t0 += kTile) {
    const int rows = min(kTile, n_kv - t0);
    const TileRows src = tile_rows(a, unit, head, sp.lo, t0);
    __syncthreads();
    load_tile<4, false>(src.k, a.k_stride, rows, kt, wave, lane);
    load_tile<4, true>(src.v, a.v_stride, rows, vt, wave, lane);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    floatx16_t s[2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      s[mt] = floatx16_t{0.f};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint4 kk = lds_read16(kr + mt * 32 * kRowBytes + (((2 * k + h) ^ (n & 15)) << 4));
        s[mt] = mfma_32x32x16<DT>(kk, q[k], s[mt]);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = t0 + mt * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
        s[mt][i] = t < lim ? s[mt][i] : -INFINITY;
        mx = fmaxf(mx, s[mt][i]);
      }
    mx = halves_max(mx);
    const float top = rounded_product(mx, c) - kBias;
    if (__any(top > (large ? m : m + 8.f))) {
      const float mn = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
      large = __any(fabsf(m) >= kLargeScaled);
    }
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float e = fmaf(s[mt][i], c, -m);
        if (large) e = rounded_product(s[mt][i], c) - m;
        s[mt][i] = __builtin_amdgcn_exp2f(e);
        l += s[mt][i];
      }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const floatx16_t& p = s[t >> 1];
      const int i = 8 * (t & 1);
      const uint4 pb = make_uint4(pack2<DT>(p[i], p[i + 1]), pack2<DT>(p[i + 2], p[i + 3]), pack2<DT>(p[i + 4], p[i + 5]),
                                  pack2<DT>(p[i + 6], p[i + 7]));
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
        const lds_char* at = vr + t * 16 * kRowBytes + (((2 * ct + g1) ^ (2 * r4 + h)) << 5);
        const uint2 v0 = lds_read_transposed(at), v1 = lds_read_transposed(at + 8 * kRowBytes);
        o[ct] = mfma_32x32x16<DT>(make_uint4(v0.x, v0.y, v1.x, v1.y), pb, o[ct]);
      }
    }
  }
  l = halves_sum(l);
  if (!there) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  char* const op = a.out + ((size_t)(sp.lo + tok) * a.n_q_heads + qh) * kRowBytes + h * 8;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(op + ct * 64 + i * 16) =
          make_uint2(pack2<DT>(o[ct][4 * i] * inv, o[ct][4 * i + 1] * inv), pack2<DT>(o[ct][4 * i + 2] * inv, o[ct][4 * i + 3] * inv));
}

// FIER_ESHAPE where the grid would not fit 32 bits, else FIER_OK or FIER_EHIP.
int launch_prompt_attn(int dtype, PromptArgs a, hipStream_t st) {
  a.row_tiles = (a.max_new * a.n_rep + 127) / 128;
  const int64_t grid = (int64_t)a.units * a.row_tiles;
  if (grid == 0) return FIER_OK;
  if (grid > INT32_MAX) return FIER_ESHAPE;
  if (dtype == DT_F16)
    prompt_attn_kernel<DT_F16><<<(unsigned)grid, 256, 0, st>>>(a);
  else
    prompt_attn_kernel<DT_BF16><<<(unsigned)grid, 256, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? FIER_OK : FIER_EHIP;
}

}  // namespace fier
