// Causal attention of many new tokens per sequence: whole prompts packed one after the other (fier_prefill_attn), and
// chunks over the rows of a cache (fier_chunk_attn).
//   Token i of a sequence's n attends over the rows 0 .. first + i; first = 0 for prompts, the length before the chunk for a
// cache.  A unit (sequence, kv head) has n * n_rep query rows, row = token * n_rep + head of the group, so that the heads that
// share K and V share their tiles too.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "fier.h"
#include "fier_dev.h"
#include "fier_kernels.h"

namespace fier {

typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx2_t __attribute__((ext_vector_type(2)));

constexpr int kRowTile = 128;  // query rows per workgroup
constexpr int kSideRows = 32;  // up to here its wavefronts all hold them
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

// The larger of two, a NaN if one is (one instruction; fmaxf has to quiet its operands first).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float halves_max(float x) {
  typedef unsigned int u2_t __attribute__((ext_vector_type(2)));
  const u2_t a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(a[0]), __uint_as_float(a[1]));
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

// ---- K and V rows into LDS ----------------------------------------------------------------------------------------------
// Direct loads, 16 bytes a lane, 1 KiB (4 rows) an instruction: lane l's 16 bytes go to the instruction's LDS address + 16 l.
// The 16-byte chunks of a row are permuted so that the reads of both products meet no bank twice: K chunk c lies at c ^ (row & 15),
// V's pair of chunks p at p ^ (2 (row & 3) + (row >> 2 & 1)).
// Written as assembly, with a wait count of its own (wait_loads): the compiler takes every read of LDS for one that may need the
// loads just issued, and waited for the next tile's rows before this one's product.  Nothing is returned in a register.  The
// instruction after a write of M0 may not use it yet.
// STREAM: with the hint for data that is read once.  (M0 is named as clobbered, so that an instruction of the compiler's own that
// used it would set it anew; the compiler remarks that it does not save the register, which nobody asks it to.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool STREAM>
__device__ __forceinline__ void load_rows_to_lds(const char* base, uint32_t off, const lds_char* dst) {
  if (STREAM)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"((uint32_t)(uintptr_t)dst), "v"(off),
                 "s"(base)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"((uint32_t)(uintptr_t)dst), "v"(off),
                 "s"(base)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
// until at most N of the wavefront's loads are under way
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// every wavefront of the workgroup is here, its LDS reads done
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The lane's number anew: what is only needed after a loop need not live in registers through it.
__device__ __forceinline__ int lane_again() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// The unit's K / V rows: row t of packed prompts, or of a cache, lies at row (t's block) * block_stride + (t & mask) of k and v.
// Tiles of 32 or 64 rows start at multiples of their size, so that they lie inside a block.
template <bool CACHE>
struct UnitRows {
  const char *k, *v;
  int64_t k_stride, v_stride;  // bytes
  // the sequence's block list, in the address space of data that no kernel writes meanwhile: it is read with scalar loads, whose
  // results are the same in all lanes without a vector load between those of the tiles
  const __attribute__((address_space(4))) int32_t* blocks;
  size_t block_stride;
  int shift, mask;
  __device__ __forceinline__ UnitRows(const PromptArgs& a, int unit, int head, int lo)
      : k(a.k), v(a.v), k_stride(CACHE ? kRowBytes : a.k_stride), v_stride(CACHE ? kRowBytes : a.v_stride), blocks(nullptr),
        block_stride(0), shift(0), mask(-1) {
    if (CACHE) {
      const KvRows c = a.lay.rows_of(unit);
      k += c.base * kRowBytes;
      v += c.base * kRowBytes;
      if (c.blocks) {
        blocks = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)c.blocks;
        block_stride = c.block_stride, shift = c.shift, mask = c.mask;
      }
    } else {
      k += (int64_t)lo * k_stride + head * kRowBytes;
      v += (int64_t)lo * v_stride + head * kRowBytes;
    }
  }
  __device__ __forceinline__ int block_of(int t) const { return CACHE && blocks ? blocks[t >> shift] : 0; }
  __device__ __forceinline__ size_t row(int block, int t) const {
    return CACHE ? (size_t)block * block_stride + (size_t)(t & mask) : (size_t)t;
  }
};

// A wavefront's share of a tile: N instructions, rows 4 (n0 + STEP j) .. + 3 of instruction j.  The permutation of a row's chunks
// repeats after 16 rows (V: 8): as many offsets differ in more than the rows' distance, which goes into the scalar address.
template <bool V, int N, int STEP>
struct RowLoads {
  static constexpr int kCycle = (V ? 8 : 16) / 4 / STEP > 1 ? (V ? 8 : 16) / 4 / STEP : 1;
  uint32_t off[kCycle];
  __device__ __forceinline__ static uint32_t chunk(int row, int lane) {
    const int c = lane & 15;
    return 16u * (uint32_t)(V ? c ^ (((row & 3) << 2) | ((row >> 1) & 2)) : c ^ (row & 15));
  }
  __device__ __forceinline__ RowLoads(int n0, int lane, int64_t stride) {
#pragma unroll
    for (int j = 0; j < kCycle; ++j) {
      const int row = 4 * (n0 + STEP * j) + (lane >> 4);
      off[j] = (uint32_t)row * (uint32_t)stride + chunk(row, lane);
    }
  }
  template <bool STREAM>
  __device__ __forceinline__ void load_whole(const char* src, int64_t stride, const lds_char* dst, int n0) const {
#pragma unroll
    for (int j = 0; j < N; ++j)
      load_rows_to_lds<STREAM>(src + (int64_t)(4 * STEP * (j / kCycle * kCycle)) * stride, off[j % kCycle],
                               dst + 4 * (n0 + STEP * j) * kRowBytes);
  }
  // rows: how many the tile has; the others take the last one's (they get no weight)
  __device__ __forceinline__ void load(const char* src, int64_t stride, int rows, const lds_char* dst, int n0,
                                       bool stream = false) const {
    if (rows >= 4 * N * STEP) {
      if (stream) load_whole<true>(src, stride, dst, n0);
      else load_whole<false>(src, stride, dst, n0);
    } else {
      const int lane = lane_again();
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int row = 4 * (n0 + STEP * j) + (lane >> 4);
        load_rows_to_lds<false>(src, (uint32_t)min(row, rows - 1) * (uint32_t)stride + chunk(row, lane),
                                dst + 4 * (n0 + STEP * j) * kRowBytes);
      }
    }
  }
};

// The lane's places in a K and a V tile of 32 rows, in registers: what differs from read to read is then a constant offset.
struct LdsReads {
  const lds_char *k[8], *v[4];
  __device__ __forceinline__ LdsReads(const lds_char* kt, const lds_char* vt, int lane) {
    const int n = lane & 31, h = lane >> 5, r4 = (lane & 15) >> 2, g1 = (lane >> 4) & 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t at = (uint32_t)(uintptr_t)kt + n * kRowBytes + (((2 * i + h) ^ (n & 15)) << 4);
      asm("" : "+v"(at));  // not made anew from its parts each time
      k[i] = (const lds_char*)(uintptr_t)at;
    }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      uint32_t at = (uint32_t)(uintptr_t)vt + (4 * h + r4) * kRowBytes + (lane & 3) * 8 + (((2 * ct + g1) ^ (2 * r4 + h)) << 5);
      asm("" : "+v"(at));
      v[ct] = (const lds_char*)(uintptr_t)at;
    }
  }
};

// ---- 32 query rows of a wavefront ---------------------------------------------------------------------------------------
// S^T = K Q^T (rows = tokens, columns = query rows): lane (n, h) holds the logits of its query row n for the tokens
// 8 i + 4 h + 0..3 of every 32, which is the B operand of O^T += V^T P^T as it stands, the tokens of a product of 16 taken in
// the order 4 h, 8 + 4 h.  V^T comes out of LDS by transposing reads.  Nothing crosses lanes but the maximum over the halves.
template <int DT>
struct Rows32 {
  // fp16 weights are scaled by 2^7, so that those down to 2^-21 of the largest keep all their bits
  static constexpr float kBias = DT == DT_F16 ? 7.f : 0.f;
  static constexpr float kSlack = 8.f;  // the maximum is moved only when a weight would pass 2^(8 + bias)
  floatx16_t o[4];  // o[c][i]: channel 32 c + 8 (i / 4) + 4 h + i % 4
  float m, l;       // what is subtracted from the scaled logits; the lane's own tokens' part of the sum
  bool large;       // some row's m is beyond kLargeScaled

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = floatx16_t{0.f};
    m = -FLT_MAX, l = 0.f;
    large = false;
  }

  // Logits of 32 tokens.  at: bytes from the tiles that `r` was made for.
  __device__ __forceinline__ static floatx16_t scores(const LdsReads& r, int at, const uint4 (&q)[8]) {
    floatx16_t s = {0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k) s = mfma_32x32x16<DT>(lds_read16(r.k[k] + at), q[k], s);
    return s;
  }

  // Logits into weights, the running maximum and sum with them.  left: how many of the tokens the row attends over (only
  // looked at if masked).
  __device__ __forceinline__ void weights(floatx16_t& s, float c, bool masked, int left, int h) {
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) < left - 4 * h ? s[i] : -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = larger(mx, s[i]);
    mx = halves_max(mx);
    const float top = rounded_product(mx, c) - kBias;
    if (__any(top > (large ? m : m + kSlack))) {  // the maxima settle after a few tiles
      const float to = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
      large = __any(fabsf(m) >= kLargeScaled && m != -FLT_MAX);  // not a row that has met no token yet
    }
    // The weights take the scaled logit unrounded, which is the more accurate while logits are small.  From 2^22 on its
    // distance from the rounded maximum would be that one's rounding error: there both are rounded alike.
    if (__builtin_expect(large, 0)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(rounded_product(s[i], c) - m);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -m));
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) l += s[i];
  }

  // The weights, rounded to the K dtype (to nearest, at most half a step: 2^-8 of each with bf16, 2^-11 with fp16), times V.  Against 64
  // bits the outputs of whole prompts are off by a fifth more than with unrounded weights, whose outputs are rounded all the same (bf16
  // 1.6e-3 -> 1.9e-3 relative, fp16 2.0e-4 -> 2.3e-4); three exact parts as in the decode step would make it three products.
  __device__ __forceinline__ void add_values(const LdsReads& r, int at, const floatx16_t& p) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint4 pb = make_uint4(pack2<DT>(p[8 * t], p[8 * t + 1]), pack2<DT>(p[8 * t + 2], p[8 * t + 3]),
                                  pack2<DT>(p[8 * t + 4], p[8 * t + 5]), pack2<DT>(p[8 * t + 6], p[8 * t + 7]));
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
        const lds_char* const from = r.v[ct] + (at + t * 16 * kRowBytes);
        const uint2 v0 = lds_read_transposed(from), v1 = lds_read_transposed(from + 8 * kRowBytes);
        o[ct] = mfma_32x32x16<DT>(make_uint4(v0.x, v0.y, v1.x, v1.y), pb, o[ct]);
      }
    }
  }
};

// A mean of V lies within V's type, but rounded weights over a sum that is not can make it larger by 2^-11 (fp16): past 65520 it
// would be rounded to an infinity, and is held at the largest value.  What is an infinity or a NaN before it is rounded stays one.  (bf16
// values that large are outside what the sums can hold.)  Behind a branch that ordinary values never take: with three instructions for
// every value a prompt of 100 tokens took 7.5 us instead of 7.3.
template <int DT, int N>
__device__ __forceinline__ void hold_overflows(float (&o)[N]) {
  constexpr float kMost = 65504.f;
  if (DT != DT_F16) return;
  float mx = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) mx = fmaxf(mx, fabsf(o[i]));
  if (__builtin_expect(__any(mx > kMost), 0)) {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = __builtin_isfinite(o[i]) ? __builtin_amdgcn_fmed3f(o[i], -kMost, kMost) : o[i];
  }
}
template <int DT>
__device__ __forceinline__ void store_channels(char* out_row, int ct, int h, const floatx16_t& o, float inv) {
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = o[i] * inv;
  hold_overflows<DT>(y);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<uint2*>(out_row + ct * 64 + i * 16 + h * 8) =
        make_uint2(pack2<DT>(y[4 * i], y[4 * i + 1]), pack2<DT>(y[4 * i + 2], y[4 * i + 3]));
}

// ---- one query row per lane and half ------------------------------------------------------------------------------------
struct QueryRow {
  const char* q;
  char* out;
  int lim;     // cache rows it attends over
  bool there;  // false: a copy of the last row, which nobody stores
  __device__ __forceinline__ QueryRow(const PromptArgs& a, const PromptSpan& sp, int head, int row, int n_rows) {
    there = row < n_rows;
    row = there ? row : n_rows - 1;
    const int tok = a.token_of(row), qh = head * a.n_rep + row - tok * a.n_rep;
    lim = min(sp.first + tok + 1, a.kv_cap);
    q = a.q + (size_t)(sp.lo + tok) * a.q_stride + qh * kRowBytes;
    out = a.out + ((size_t)(sp.lo + tok) * a.n_q_heads + qh) * kRowBytes;
  }
};

// ---- partial results of side-by-side parts ---------------------------------------------------------------------------------
// o of 32 query rows as the lanes hold it (four channel tiles of 16 floats a lane), then m and l of every lane.  Written through to
// memory and read past the caches: another workgroup of the launch reads them (see arrive_add).  Only lanes whose row is there
// take part: with one token of four heads an eighth of them.
constexpr int kPartFloats = 32 * kD + 2 * 64;
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
  return (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32;
}
__device__ __forceinline__ float low_of(unsigned long long w) { return __uint_as_float((uint32_t)w); }
__device__ __forceinline__ float high_of(unsigned long long w) { return __uint_as_float((uint32_t)(w >> 32)); }
__device__ __forceinline__ void store_partial(float* slot, int ct, const floatx16_t& o, float m, float l, int lane) {
  unsigned long long* const p = reinterpret_cast<unsigned long long*>(slot + ct * 1024) + lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) store_coherent(p + i * 64, pair_of(o[2 * i], o[2 * i + 1]));
  if (ct == 0) store_coherent(reinterpret_cast<unsigned long long*>(slot + 32 * kD) + lane, pair_of(m, l));
}
// Channel tile ct of n slots, `pitch` floats apart, joined, the loads of eight under way together.
__device__ __forceinline__ void join_partials(const float* slots, size_t pitch, int n, int ct, int lane, floatx16_t& o, float& m,
                                              float& l) {
  constexpr int kBatch = 8;
  m = -FLT_MAX, l = 0.f;
  o = floatx16_t{0.f};
  for (int p0 = 0; p0 < n; p0 += kBatch) {
    unsigned long long ml[kBatch], w[kBatch][8];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float* const slot = slots + (size_t)min(p0 + k, n - 1) * pitch;
      ml[k] = load_coherent(reinterpret_cast<const unsigned long long*>(slot + 32 * kD) + lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[k][i] = load_coherent(reinterpret_cast<const unsigned long long*>(slot + ct * 1024) + i * 64 + lane);
    }
    float to = m;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) to = fmaxf(to, low_of(ml[k]));
    const float alpha = __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= alpha;
    o *= alpha;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float f = p0 + k < n ? __builtin_amdgcn_exp2f(low_of(ml[k]) - m) : 0.f;
      l += f * high_of(ml[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[2 * i] += f * low_of(w[k][i]), o[2 * i + 1] += f * high_of(w[k][i]);
    }
  }
}

// ---- which workgroup does what -----------------------------------------------------------------------------------------------
// A sequence's query rows per kv head are cut into tiles of 128; the last one, where it has at most 32, goes through its K / V
// rows side by side, the others share them.  Over a cache the K / V rows of a tile are split into parts of `step` steps, one length
// for all sequences of the call, so that unequal ones keep the GPU busy to the end: `step` is the call's steps over the
// number of parts wanted, about as many as the GPU holds workgroups of this kernel at once (256 CUs x 3).  Lengths lie on the GPU,
// so every workgroup works this out for itself, one sequence a lane.  us with one number of parts for all sequences / this: chunks
// of 1 to 500 tokens of 8 sequences of up to 12000, 24 q / 8 kv heads 458 / 270; one token of 16 sequences of 8k-64k 531 / 485.
constexpr int kSideTile = 32;    // rows of K and V per wavefront and step side by side
constexpr int kSideWaves = 3;    // of the four: so three such workgroups fit a CU's LDS
constexpr int kSideStep = kSideWaves * kSideTile;
constexpr int kSideLeast = 1;    // steps of a part, at least
constexpr int kSharedLeast = 2;  // steps of 64 rows of a part of shared rows, at least
// Parts of a tile, at most.  Side by side, up to 8 are joined by the last of their workgroups; more in groups of up to 7 by the last of
// each, and the groups by the last of those: eight counters.  Up to 64 steps are not worth the second round: 2 x 2000 tokens, 8 kv heads
// 16.0 us in 11 parts, 12.0 in 8.
constexpr int kGroup = 8, kMostParts = 48;
constexpr int kPartsWanted = 768;
// From so many bytes of K and V on, more than the last cache keeps, side-by-side tiles are loaded with the streaming hint.  One token, us
// without / with it, the rows read by other calls in between and, in parentheses, by the same call before:
//   1 sequence, 32 q / 8 kv heads      128 MiB 41.6 / 41.0 (35.3 / 38.2)   256 MiB 66.3 / 61.5 (55.5 / 60.0)   512 MiB 115 / 105 (114 / 103)
//   8 sequences, 32 heads               64 MiB 25.7 / 28.4 (22.9 / 24.4)   128 MiB 38.0 / 39.6 (33.3 / 41.2)
//                                      256 MiB 61.2 / 60.0 (52.1 / 62.9)   512 MiB 109 / 101 (110 / 101)
// and 16 sequences of 8k-64k (2.8 GB) 528 / 484.
constexpr float kStreamBytes = 256 << 20;
constexpr unsigned kGridY = 32768;  // items along y, the rest along z

struct SequenceWork {
  PromptSpan sp;
  int n_rows, tiles, aside;  // tiles of shared rows; rows of the side-by-side tile or 0
  int n_kv;                  // rows of K and V that the last query row attends over
  // tokens: of the sequences in front of the lanes' ones, 64 more of them afterwards.  Offsets that do not ascend can make
  // sequences share tokens: those with which there would be more than n_tokens of them in all count as empty, so that the grid
  // always holds every item and no split tile is left without one of its parts.
  __device__ __forceinline__ SequenceWork(const PromptArgs& a, int b, int lane, int64_t& tokens) {
    sp = PromptSpan{0, 0, 0};
    if (b < a.batch) sp = a.span(b);
    const uint32_t upto = wave_incl_scan_u32((uint32_t)sp.n, lane);
    if (tokens + upto > (int64_t)a.n_tokens) sp.n = 0;
    tokens += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    n_rows = sp.n * a.n_rep;
    const int rest = n_rows % kRowTile;
    aside = rest <= kSideRows ? rest : 0;
    tiles = n_rows / kRowTile + (rest > kSideRows ? 1 : 0);
    n_kv = min(sp.first + sp.n, a.kv_cap);
  }
  template <bool SIDE>
  __device__ __forceinline__ int steps() const {  // of the last tile
    return SIDE ? (n_kv + kSideStep - 1) / kSideStep : (n_kv + kTile - 1) / kTile;
  }
  template <bool SIDE>
  __device__ __forceinline__ int parts(int step) const {  // that its last tile has
    const int n = steps<SIDE>();
    return n <= step ? 1 : min((n + step - 1) / step, SIDE && n <= kGroup * kGroup ? kGroup : kMostParts);
  }
};
struct Item {
  PromptSpan sp;
  int b, at;    // sequence; which of its items
  int parts;    // of its tiles
  int step;     // steps of a part
  int slot;     // partial results: the place of the sequence's first item
  bool stream;  // K and V are loaded with the streaming hint
};
// Sum of the lanes' values, the same in every lane and workgroup.
__device__ __forceinline__ float wave_sum_ordered(float x) {
  x += row_ror<8>(x), x += row_ror<4>(x), x += row_ror<2>(x), x += row_ror<1>(x);
  const int v = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(v, 0)) + __int_as_float(__builtin_amdgcn_readlane(v, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(v, 32)) + __int_as_float(__builtin_amdgcn_readlane(v, 48)));
}
// Where part p of n begins: all <= 2^14 steps, p <= n <= 48.
__device__ __forceinline__ int part_begin(int all, int p, int n) { return (int)((unsigned)(all * p) / (unsigned)n); }
// Item number j of the launch's (per kv head); false: there are fewer.
template <bool SIDE, bool SPLIT>
__device__ __forceinline__ bool find_item(const PromptArgs& a, int j, int lane, Item& it) {
  int64_t tokens0 = 0;
  const SequenceWork w0(a, lane, lane, tokens0);  // more than 64 sequences: the others are looked at in turn
  it.step = 1 << 30;
  it.stream = false;
  if (SPLIT) {
    // steps of all tiles, and (shared) tiles
    float all = 0.f, tiles = 0.f;
    auto count = [&](const SequenceWork& w) {
      const float n = (float)(SIDE ? (w.aside ? 1 : 0) : w.tiles);
      all += wave_sum_ordered(n * (float)w.steps<SIDE>());
      if (!SIDE) tiles += wave_sum_ordered(n);
    };
    count(w0);
    int64_t tokens = tokens0;
    for (int b0 = 64; b0 < a.batch; b0 += 64) count(SequenceWork(a, b0 + lane, lane, tokens));
    // A tile of s steps becomes ceil(s / step) items, half of one more than s / step on average.  Shared tiles take the GPU for
    // long: their items are to fit one round, two where the tiles alone fill more than half of one; many tiles are split where one
    // has more than its share of two rounds.  us in one round / two, 32 q / 8 kv heads behind 32768 tokens (32 heads behind 4096 in
    // parentheses), tiles over places: 0.49 813 / 816 (138 / 155), 0.54 1124 / 949 (235 / 172), 0.62 1147 / 1046; two rounds less the
    // halves / two rounds: 1.1 1915 / 1918 (350 / 411), 1.3 2883 / 2137 (453 / 473).
    float wanted = (float)a.parts_wanted;
    if (!SIDE) wanted = tiles > 1.2f * wanted ? 2.f * wanted : (tiles > 0.5f * wanted ? 2.f : 1.f) * wanted - 0.5f * tiles;
    it.step = __builtin_amdgcn_readfirstlane(max(SIDE ? kSideLeast : kSharedLeast, (int)ceilf(all / wanted)));
    it.stream = all * (float)a.n_kv_heads * (2.f * kSideStep * kRowBytes) >= kStreamBytes;
  }
  int before = 0, slots = 0;
  auto look = [&](const SequenceWork& w, int b0) {
    const int parts = SPLIT ? w.parts<SIDE>(it.step) : 1, n = (SIDE ? (w.aside ? 1 : 0) : w.tiles) * parts;
    const int split = parts > 1 ? n : 0;
    const int upto = before + (int)wave_incl_scan_u32((uint32_t)n, lane);
    const int slots_upto = SPLIT ? slots + (int)wave_incl_scan_u32((uint32_t)split, lane) : 0;
    const unsigned long long past = __ballot(upto > j);
    if (past) {
      const int l = __builtin_ctzll(past);
      it.b = b0 + l;
      it.sp = PromptSpan{__builtin_amdgcn_readlane(w.sp.lo, l), __builtin_amdgcn_readlane(w.sp.n, l), __builtin_amdgcn_readlane(w.sp.first, l)};
      it.at = j - __builtin_amdgcn_readlane(upto - n, l);
      it.parts = __builtin_amdgcn_readlane(parts, l);
      it.slot = __builtin_amdgcn_readlane(slots_upto - split, l);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
    slots = __builtin_amdgcn_readlane(slots_upto, 63);
    return false;
  };
  if (look(w0, 0)) return true;
  for (int b0 = 64; b0 < a.batch; b0 += 64)
    if (look(SequenceWork(a, b0 + lane, lane, tokens0), b0)) return true;
  return false;
}

// Part `part` of n_parts is done: its partial results (channel tile `wave` of the lanes that are there) go to its slot, and the last
// workgroup of all returns true with those of all parts joined in o, m and l.
__device__ __forceinline__ bool join_parts(float* slots, int n_parts, int part, uint32_t* counters, bool there, int wave, int lane,
                                           floatx16_t& o, float& m, float& l, uint32_t* flag) {
  const bool first = wave == 0 && lane == 0;
  if (there) store_partial(slots + (size_t)part * kPartFloats, wave, o, m, l, lane);
  int group = 1, n = n_parts;  // parts per group, groups
  if (n_parts > kGroup) {
    group = 3;
    while (group * group < n_parts) ++group;  // at most 7
    n = (n_parts + group - 1) / group;
    const int g = part / group, size = min(group, n_parts - g * group);
    if (arrive_add(counters + 1 + g, 1u, flag, first) != (uint32_t)size - 1) return false;
    float* const mine = slots + (size_t)(g * group) * kPartFloats;  // the group's first slot takes the group's results
    if (there) join_partials(mine, kPartFloats, size, wave, lane, o, m, l);
    wait_loads<0>();
    meet();  // every wavefront has read the sums there
    if (there) store_partial(mine, wave, o, m, l, lane);
    if (first) store_coherent(counters + 1 + g, 0u);
  }
  if (arrive_add(counters, 1u, flag, first) != (uint32_t)n - 1) return false;
  if (there) join_partials(slots, (size_t)group * kPartFloats, n, wave, lane, o, m, l);
  if (first) store_coherent(counters, 0u);
  return true;
}

// The wavefronts' results of a side-by-side tile: each puts its own into its LDS, then takes one channel tile of all.
template <int DT, bool CACHE>
__device__ __forceinline__ void join_side_by_side(const PromptArgs& a, const Item& it, int head, const Rows32<DT>& st, int wave,
                                                  lds_char* lds, uint32_t* flag) {
  const int lane = lane_again(), h = lane >> 5;
  const int unit = it.b * a.n_kv_heads + head, n_rows = it.sp.n * a.n_rep;
  const QueryRow row(a, it.sp, head, n_rows / kRowTile * kRowTile + (lane & 31), n_rows);
  const float l = halves_sum(st.l);
  typedef __attribute__((address_space(3))) float lds_float;
  typedef float f2_t __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) f2_t lds_f2;
  lds_f2* const ml = (lds_f2*)(lds + 2 * kSideStep * kRowBytes);
  if (wave < kSideWaves) {
    lds_float* const mine = (lds_float*)(lds + wave * 2 * kSideTile * kRowBytes);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[(ct * 16 + i) * 64 + lane] = st.o[ct][i];
    ml[wave * 64 + lane] = f2_t{st.m, l};
  }
  meet();
  float m = -FLT_MAX, sum = 0.f;
  f2_t of[kSideWaves];
#pragma unroll
  for (int w = 0; w < kSideWaves; ++w) {
    of[w] = ml[w * 64 + lane];
    m = fmaxf(m, of[w].x);
  }
  floatx16_t o = {0.f};
#pragma unroll
  for (int w = 0; w < kSideWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(of[w].x - m);
    sum += f * of[w].y;
    const lds_float* const p = (const lds_float*)(lds + w * 2 * kSideTile * kRowBytes);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] += f * p[(wave * 16 + i) * 64 + lane];
  }
  if (CACHE && it.parts > 1 &&
      !join_parts(a.side_partials + ((size_t)head * a.side_slots + it.slot) * kPartFloats, it.parts, it.at,
                  a.counters + (size_t)unit * kSelBins, row.there, wave, lane, o, m, sum, flag))
    return;
  if (row.there) store_channels<DT>(row.out, wave, h, o, sum > 0.f ? 1.f / sum : 0.f);
}

// Up to 32 query rows: three wavefronts hold them all and go side by side through the K / V rows, each through 32 of every 96, in
// 16 KiB of LDS of its own, so that nobody waits for anybody.  The next K rows are loaded once this step's logits are there, the
// next V rows after its product.  Bound by memory: nine wavefronts with 8 to 16 KiB under way each on a CU.
template <int DT, bool CACHE>
__device__ __forceinline__ void attend_side_by_side(const PromptArgs& a, const Item& it, int head, lds_char* lds, uint32_t* flag) {
  const PromptSpan sp = it.sp;
  const int unit = it.b * a.n_kv_heads + head, n_rows = sp.n * a.n_rep, row0 = n_rows / kRowTile * kRowTile;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int n_kv = min(sp.first + sp.n, a.kv_cap);
  const int all = (n_kv + kSideStep - 1) / kSideStep, n_parts = it.parts;
  const int begin = CACHE ? part_begin(all, it.at, n_parts) : 0, end = CACHE ? part_begin(all, it.at + 1, n_parts) : all;
  const QueryRow row(a, sp, head, row0 + n, n_rows);
  const int least = __builtin_amdgcn_readfirstlane(row.lim);  // the first row's
  const UnitRows<CACHE> rows(a, unit, head, sp.lo);
  lds_char* const kt = lds + wave * 2 * kSideTile * kRowBytes;
  lds_char* const vt = kt + kSideTile * kRowBytes;
  const LdsReads reads(kt, vt, lane);
  const RowLoads<false, 8, 1> kl(0, lane, rows.k_stride);
  const RowLoads<true, 8, 1> vl(0, lane, rows.v_stride);
  int t0 = begin * kSideStep + wave * kSideTile;
  const int stop = wave < kSideWaves ? min(end * kSideStep, n_kv) : 0;
  int block = 0;
  if (t0 < stop) {
    const size_t r = rows.row(rows.block_of(t0), t0);
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - t0, kt, 0, it.stream);
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - t0, vt, 0, it.stream);
    block = rows.block_of(t0 + kSideStep < stop ? t0 + kSideStep : t0);
  }
  uint4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = a.load_q(row.q + s * 32 + h * 16);
  Rows32<DT> st;
  st.init();
  for (; t0 < stop; t0 += kSideStep) {
    const int next = t0 + kSideStep < stop ? t0 + kSideStep : t0;  // the last step loads its own rows once more
    const size_t r = rows.row(block, next);
    wait_loads<8>();
    floatx16_t s = Rows32<DT>::scores(reads, 0, q);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - next, kt, 0, it.stream);
    block = rows.block_of(next + kSideStep < stop ? next + kSideStep : next);  // for the step after the next: the list is far away
    st.weights(s, a.scale, t0 + kSideTile > least, row.lim - t0, h);
    wait_loads<8>();
    st.add_values(reads, 0, s);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - next, vt, 0, it.stream);
  }
  wait_loads<0>();
  join_side_by_side<DT, CACHE>(a, it, head, st, wave, lds, flag);
}

// Which tile and part of a sequence's shared rows an item is; the tiles that attend over the most rows come first.
struct SharedTile {
  int tiles, turned, tile, part, n_kv, all, n_parts;  // n_kv rows, `all` steps; a prompt's first tiles have fewer than the last
  __device__ __forceinline__ SharedTile(const PromptArgs& a, const Item& it) {
    const int n_rows = it.sp.n * a.n_rep;
    tiles = n_rows / kRowTile + (n_rows % kRowTile > kSideRows ? 1 : 0);
    turned = it.parts > 1 ? it.at / it.parts : it.at;
    part = it.at - turned * it.parts;
    tile = tiles - 1 - turned;
    n_kv = min(it.sp.first + a.token_of(min((tile + 1) * kRowTile, n_rows) - 1) + 1, a.kv_cap);
    all = (n_kv + kTile - 1) / kTile;
    n_parts = it.parts > 1 ? min(it.parts, (all + it.step - 1) / it.step) : 1;
  }
};

// ---- shared tiles in several parts: a second launch joins them ------------------------------------------------------------------
// Joined by the last workgroup of each tile, as the side-by-side ones are, it was one CU that read up to 3 MB: 64 tokens of 32 q / 8 kv
// heads behind 32768 took 93 us, now 56 with the rows in the last cache and 69 without.  (Still twice what the bytes need: 94 partial
// results a head of 67.6 KB each, 51 MB written and read again beside 134 MB of K and V.)
// Per wavefront o as the lanes hold it, 16 chunks of 64 x 4 floats (channel tile ct, channels 8 i + 4 h + 0..3: chunk 4 ct + i),
// then m and l of the lanes.
__device__ __forceinline__ float* shared_slot(const PromptArgs& a, const Item& it, int head, int turned, int part) {
  return a.shared_partials + ((size_t)head * a.shared_slots + it.slot + turned * it.parts + part) * (4 * kPartFloats);
}
template <int DT, bool CACHE>
__device__ __forceinline__ void finish_shared(const PromptArgs& a, const Item& it, int head, int tiles, int turned, int part, int n_parts,
                                              const Rows32<DT>& st, int wave) {
  const int lane = lane_again(), h = lane >> 5;
  const float l = halves_sum(st.l);
  if (CACHE && n_parts > 1) {
    float4* const p = reinterpret_cast<float4*>(shared_slot(a, it, head, turned, part) + wave * kPartFloats) + lane;
#pragma unroll
    for (int c = 0; c < 16; ++c)
      p[c * 64] = make_float4(st.o[c >> 2][4 * (c & 3)], st.o[c >> 2][4 * (c & 3) + 1], st.o[c >> 2][4 * (c & 3) + 2], st.o[c >> 2][4 * (c & 3) + 3]);
    reinterpret_cast<float2*>(p - lane + 16 * 64)[lane] = make_float2(st.m, l);
    return;
  }
  const QueryRow row(a, it.sp, head, (tiles - 1 - turned) * kRowTile + wave * 32 + (lane & 31), it.sp.n * a.n_rep);
  if (!row.there) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) store_channels<DT>(row.out, ct, h, st.o[ct], inv);
}

// CH chunks of a wavefront's 32 rows at a time, BATCH parts' loads under way together.
template <int DT, int CH, int BATCH>
__device__ __forceinline__ void join_chunks(const PromptArgs& a, const Item& it, int head, const SharedTile& t, int first, int lane) {
  for (int c = first * CH; c < 64; c += 4 * CH * t.n_parts) {
    const float* const from = shared_slot(a, it, head, t.turned, 0) + (c >> 4) * kPartFloats;
    float m = -FLT_MAX, l = 0.f, o[CH][4] = {};
    for (int p0 = 0; p0 < t.n_parts; p0 += BATCH) {
      float4 w[BATCH][CH];
      float2 ml[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const float4* const slot = reinterpret_cast<const float4*>(from + (size_t)min(p0 + k, t.n_parts - 1) * (4 * kPartFloats));
#pragma unroll
        for (int x = 0; x < CH; ++x) w[k][x] = slot[((c & 15) + x) * 64 + lane];
        ml[k] = reinterpret_cast<const float2*>(slot + 16 * 64)[lane];
      }
      float to = m;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) to = fmaxf(to, ml[k].x);
      const float alpha = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= alpha;
#pragma unroll
      for (int x = 0; x < CH; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[x][i] *= alpha;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const float f = p0 + k < t.n_parts ? __builtin_amdgcn_exp2f(ml[k].x - m) : 0.f;
        l += f * ml[k].y;
#pragma unroll
        for (int x = 0; x < CH; ++x)
          o[x][0] += f * w[k][x].x, o[x][1] += f * w[k][x].y, o[x][2] += f * w[k][x].z, o[x][3] += f * w[k][x].w;
      }
    }
    const QueryRow row(a, it.sp, head, t.tile * kRowTile + (c >> 4) * 32 + (lane & 31), it.sp.n * a.n_rep);
    const float inv = l > 0.f ? 1.f / l : 0.f;
    float y[4 * CH];
#pragma unroll
    for (int x = 0; x < CH; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[4 * x + i] = o[x][i] * inv;
    hold_overflows<DT>(y);
    if (row.there) {
#pragma unroll
      for (int x = 0; x < CH; ++x)
        *reinterpret_cast<uint2*>(row.out + ((c & 15) + x) * 16 + (lane >> 5) * 8) =
            make_uint2(pack2<DT>(y[4 * x], y[4 * x + 1]), pack2<DT>(y[4 * x + 2], y[4 * x + 3]));
    }
  }
}
// One workgroup for every part of the first launch; a tile's share the 64 chunks of its rows.
template <int DT>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = (int)(blockIdx.z * kGridY + blockIdx.y), head = (int)blockIdx.x;
  Item it;
  if (!find_item<false, true>(a, j, lane, it) || it.parts == 1) return;
  const SharedTile t(a, it);
  if (t.part >= t.n_parts || t.n_parts == 1) return;
  // The fewer the parts, the more chunks a wavefront has: 16 loads under way in any case.
  const int first = t.part * 4 + wave;
  if (t.n_parts <= 2) join_chunks<DT, 8, 2>(a, it, head, t, first, lane);
  else if (t.n_parts <= 4) join_chunks<DT, 4, 4>(a, it, head, t, first, lane);
  else if (t.n_parts <= 8) join_chunks<DT, 2, 8>(a, it, head, t, first, lane);
  else join_chunks<DT, 1, 16>(a, it, head, t, first, lane);
}

// 128 query rows, 32 a wavefront; the K / V rows go through LDS 64 at a time, shared by the wavefronts: two tiles of K, whose next
// one is loaded a step ahead, and one of V, loaded during the step's first logits.  48 KiB and at most 168 registers, so that
// three workgroups share a CU and one's products run beside another's exponentials.
//   What bounds it: power.  At 16384 tokens of 32 heads (2.09 ms, 1.05 PFLOP/s; a large library product of random numbers makes
// 1.2) the matrix cores are busy 62 % of the cycles, at 1.6 GHz; without the softmax the loop runs at 1.22.  Two workgroups per
// CU with twice the registers, each wavefront's exponentials interleaved with its next products, were busy 50 % at 1.74 GHz:
// 2.30 ms.  64 rows a wavefront (half the LDS reads) needs accumulation registers and the moves to and from them: 2.83.  Fewer
// instructions pay: addresses in registers instead of made anew 2.16 -> 2.09.
template <int DT, bool CACHE>
__device__ __forceinline__ void attend_shared(const PromptArgs& a, const Item& it, int head, lds_char* lds) {
  const PromptSpan sp = it.sp;
  const int unit = it.b * a.n_kv_heads + head, n_rows = sp.n * a.n_rep;
  const SharedTile t(a, it);
  const int part = t.part, n_parts = t.n_parts, n_kv = t.n_kv, all = t.all, row0 = t.tile * kRowTile;
  if (CACHE && part >= n_parts) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int begin = CACHE ? part_begin(all, part, n_parts) : 0, end = CACHE ? part_begin(all, part + 1, n_parts) : all;
  const QueryRow row(a, sp, head, row0 + wave * 32 + n, n_rows);
  const int least = __builtin_amdgcn_readfirstlane(row.lim), most = __builtin_amdgcn_readlane(row.lim, 31);
  const UnitRows<CACHE> rows(a, unit, head, sp.lo);
  constexpr int kBytes = kTile * kRowBytes;
  const RowLoads<false, 4, 4> kl(wave, lane, rows.k_stride);
  const RowLoads<true, 4, 4> vl(wave, lane, rows.v_stride);
  const size_t r0 = rows.row(rows.block_of(begin * kTile), begin * kTile);
  kl.load(rows.k + r0 * rows.k_stride, rows.k_stride, n_kv - begin * kTile, lds, wave);
  size_t r = r0;
  int block = rows.block_of(min(begin + 1, end - 1) * kTile);
  uint4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = a.load_q(row.q + s * 32 + h * 16);
  Rows32<DT> st;
  st.init();
  lds_char* const vt = lds + 2 * kBytes;
  const LdsReads reads(lds, vt, lane);
  // Tile i, its K rows in the buffer CUR: a constant, so that it goes into the reads' offsets.
  auto step = [&](int i, auto CUR) {
    constexpr int cur = decltype(CUR)::value;
    const int t0 = i * kTile, next = i + 1 < end ? t0 + kTile : t0;
    wait_loads<0>();
    meet();
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - t0, vt, wave);
    r = rows.row(block, next);
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - next, lds + (cur ^ 1) * kBytes, wave);
    block = rows.block_of(min(i + 2, end - 1) * kTile);
    floatx16_t s;
    if (t0 < most) {  // some of the wavefront's rows go that far
      s = Rows32<DT>::scores(reads, cur * kBytes, q);
      st.weights(s, a.scale, t0 + 32 > least, row.lim - t0, h);
    }
    wait_loads<4>();
    meet();
    if (t0 < most) st.add_values(reads, 0, s);
    if (t0 + 32 < most) {
      s = Rows32<DT>::scores(reads, cur * kBytes + 32 * kRowBytes, q);
      st.weights(s, a.scale, t0 + kTile > least, row.lim - t0 - 32, h);
      st.add_values(reads, 32 * kRowBytes, s);
    }
  };
  for (int i = begin; i < end; i += 2) {
    step(i, std::integral_constant<int, 0>());
    if (i + 1 < end) step(i + 1, std::integral_constant<int, 1>());
  }
  wait_loads<0>();
  finish_shared<DT, CACHE>(a, it, head, t.tiles, t.turned, part, n_parts, st, wave);
}

// The grid lists the side-by-side items first, then the shared ones, the kv heads of an item next to each other: with a multiple
// of 8 of them a head's K and V stay in one XCD's L2.  What has no work leaves at once.
//   CACHE: over a cache's rows, split where there are few tiles; else packed prompts, not split.
template <int DT, bool CACHE>
__global__ __launch_bounds__(256, 3) void prompt_attn_kernel(PromptArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[3 * kTile * kRowBytes + kSideWaves * 64 * 8];
  __shared__ uint32_t flag;
  const int lane = threadIdx.x & 63;
  const int j = (int)(blockIdx.z * kGridY + blockIdx.y), head = (int)blockIdx.x;
  Item it;
  if (j < a.side_items) {
    if (find_item<true, CACHE>(a, j, lane, it)) attend_side_by_side<DT, CACHE>(a, it, head, (lds_char*)lds, &flag);
  } else {
    if (find_item<false, CACHE>(a, j - a.side_items, lane, it)) attend_shared<DT, CACHE>(a, it, head, (lds_char*)lds);
  }
}

// How the launch is cut.
PromptSplit prompt_split(int batch, int n_kv_heads, int n_rep, int n_tokens, int max_new, bool split) {
  PromptSplit sp = {};
  const int64_t rows = (int64_t)max_new * n_rep, all_rows = (int64_t)n_tokens * n_rep;
  const int64_t seqs = std::min(batch, n_tokens), tiles = all_rows / kRowTile + seqs;
  const bool shared = rows > kSideRows;  // some sequence may have more rows than go side by side
  sp.parts = split ? std::max(1, kPartsWanted / n_kv_heads) : 0;
  // Items: fewer than steps / step + 1 of every tile; shared tiles want up to twice the parts.
  sp.side_items = seqs + sp.parts;
  sp.shared_items = shared ? tiles + 2 * sp.parts : 0;
  // Those of tiles in several parts: ceil(x) < 2 x for x > 1.
  sp.side_slots = (int)std::min<int64_t>(2 * sp.parts, seqs * kMostParts);
  sp.shared_slots = shared ? (int)std::min<int64_t>(4 * sp.parts, tiles * kMostParts) : 0;
  sp.side_floats = (size_t)sp.side_slots * n_kv_heads * kPartFloats;
  sp.shared_floats = (size_t)sp.shared_slots * n_kv_heads * 4 * kPartFloats;
  return sp;
}

// FIER_ESHAPE where the grid would not fit 32 bits, else FIER_OK or FIER_EHIP.
int launch_prompt_attn(int dtype, PromptArgs a, const PromptSplit& sp, hipStream_t st) {
  const int64_t items = sp.side_items + sp.shared_items;
  if (a.max_new == 0) return FIER_OK;
  if (items * a.n_kv_heads > INT32_MAX) return FIER_ESHAPE;
  a.side_items = (int)sp.side_items;
  a.parts_wanted = sp.parts;
  a.side_slots = sp.side_slots, a.shared_slots = sp.shared_slots;
  a.shared_partials = a.side_partials + sp.side_floats;
  auto over = [&](int64_t n) {
    return dim3((unsigned)a.n_kv_heads, (unsigned)std::min<int64_t>(n, kGridY), (unsigned)((n + kGridY - 1) / kGridY));
  };
  const dim3 grid = over(items), join = over(sp.shared_items);
  const bool cache = a.seq_lens != nullptr;
#define FIER_PROMPT(DT)                                              \
  if (cache) prompt_attn_kernel<DT, true><<<grid, 256, 0, st>>>(a);  \
  else prompt_attn_kernel<DT, false><<<grid, 256, 0, st>>>(a);       \
  if (sp.shared_slots) prompt_join_kernel<DT><<<join, 256, 0, st>>>(a)
  if (dtype == DT_F16) {
    FIER_PROMPT(DT_F16);
  } else {
    FIER_PROMPT(DT_BF16);
  }
#undef FIER_PROMPT
  return hipGetLastError() == hipSuccess ? FIER_OK : FIER_EHIP;
}

}  // namespace fier
