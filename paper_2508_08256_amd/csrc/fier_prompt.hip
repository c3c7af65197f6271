// Causal attention of many new tokens per sequence: whole prompts packed one after the other (fier_prefill_attn), and
// chunks over the rows of a cache (fier_chunk_attn).
//   Token i of a sequence's n attends over the rows 0 .. first + i; first = 0 for prompts, the length before the chunk for a
// cache.  A unit (sequence, kv head) has n * n_rep query rows, row = token * n_rep + head of the group, so that the heads that
// share K and V share their tiles too.
#include <float.h>

#include <algorithm>

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

// ---- K and V rows into LDS ----------------------------------------------------------------------------------------------
// Direct loads, 16 bytes a lane, 1 KiB (4 rows) an instruction: lane l's 16 bytes go to the instruction's LDS address + 16 l.
// The 16-byte chunks of a row are permuted so that the reads of both products meet no bank twice: K chunk c lies at c ^ (row & 15),
// V's pair of chunks p at p ^ (2 (row & 3) + (row >> 2 & 1)).
// Written as assembly, with a wait count of its own (wait_loads): the compiler takes every read of LDS for one that may need the
// loads just issued, and waited for the next tile's rows before this one's product.  Nothing is returned in a register.  The
// instruction after a write of M0 may not use it yet.
__device__ __forceinline__ void load_rows_to_lds(const char* base, uint32_t off, const lds_char* dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"((uint32_t)(uintptr_t)dst), "v"(off), "s"(base)
               : "memory");
}
// until at most N of the wavefront's loads are under way
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// every wavefront of the workgroup is here, its LDS reads done
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The unit's K / V rows: row t of packed prompts, or of a cache, lies at row (t's block) * block_stride + (t & mask) of k and v.
// Tiles of 32 or 64 rows start at multiples of their size, so that they lie inside a block.
struct UnitRows {
  const char *k, *v;
  int64_t k_stride, v_stride;  // bytes
  // the sequence's block list, in the address space of data that no kernel writes meanwhile: it is read with scalar loads, whose
  // results are the same in all lanes without a vector load between those of the tiles
  const __attribute__((address_space(4))) int32_t* blocks;
  size_t block_stride;
  int shift, mask;
  __device__ __forceinline__ UnitRows(const PromptArgs& a, int unit, int head, int lo)
      : k(a.k), v(a.v), k_stride(a.k_stride), v_stride(a.v_stride), blocks(nullptr), block_stride(0), shift(0), mask(-1) {
    if (a.from_cache) {
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
  __device__ __forceinline__ int block_of(int t) const { return blocks ? blocks[t >> shift] : 0; }
  __device__ __forceinline__ size_t row(int block, int t) const { return (size_t)block * block_stride + (size_t)(t & mask); }
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
  // rows: how many the tile has; the others take the last one's (they get no weight)
  __device__ __forceinline__ void load(const char* src, int64_t stride, int rows, const lds_char* dst, int n0, int lane) const {
    if (rows >= 4 * N * STEP) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        load_rows_to_lds(src + (int64_t)(4 * STEP * (j / kCycle * kCycle)) * stride, off[j % kCycle], dst + 4 * (n0 + STEP * j) * kRowBytes);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int row = 4 * (n0 + STEP * j) + (lane >> 4);
        load_rows_to_lds(src, (uint32_t)min(row, rows - 1) * (uint32_t)stride + chunk(row, lane), dst + 4 * (n0 + STEP * j) * kRowBytes);
      }
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

  template <int M>
  __device__ __forceinline__ static void scores(const lds_char* kt, const uint4 (&q)[8], int n, int h, floatx16_t (&s)[M]) {
    const lds_char* const kr = kt + n * kRowBytes;
#pragma unroll
    for (int mt = 0; mt < M; ++mt) {
      s[mt] = floatx16_t{0.f};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        s[mt] = mfma_32x32x16<DT>(lds_read16(kr + mt * 32 * kRowBytes + (((2 * k + h) ^ (n & 15)) << 4)), q[k], s[mt]);
    }
  }

  // Logits into weights, the running maximum and sum with them.  left: how many of the tile's tokens the row attends over
  // (only looked at if masked).
  template <int M>
  __device__ __forceinline__ void weights(floatx16_t (&s)[M], float c, bool masked, int left, int h) {
    if (masked) {
#pragma unroll
      for (int mt = 0; mt < M; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[mt][i] = mt * 32 + 8 * (i >> 2) + (i & 3) < left - 4 * h ? s[mt][i] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 16 * M; ++i) mx = fmaxf(mx, s[i >> 4][i & 15]);
    mx = halves_max(mx);
    const float top = rounded_product(mx, c) - kBias;
    if (__any(top > (large ? m : m + kSlack))) {
      const float to = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) o[ct] *= alpha;
      large = __any(fabsf(m) >= kLargeScaled);
    }
    // The weights take the scaled logit unrounded, which is the more accurate while logits are small.  From 2^22 on its
    // distance from the rounded maximum would be that one's rounding error: there both are rounded alike.
    if (__builtin_expect(large, 0)) {
#pragma unroll
      for (int i = 0; i < 16 * M; ++i) s[i >> 4][i & 15] = __builtin_amdgcn_exp2f(rounded_product(s[i >> 4][i & 15], c) - m);
    } else {
#pragma unroll
      for (int i = 0; i < 16 * M; ++i) s[i >> 4][i & 15] = __builtin_amdgcn_exp2f(fmaf(s[i >> 4][i & 15], c, -m));
    }
#pragma unroll
    for (int i = 0; i < 16 * M; ++i) l += s[i >> 4][i & 15];
  }

  template <int M>
  __device__ __forceinline__ void add_values(const lds_char* vt, const floatx16_t (&p)[M], int lane, int h) {
    const int r4 = (lane & 15) >> 2, g1 = (lane >> 4) & 1;
    const lds_char* const vr = vt + (4 * h + r4) * kRowBytes + (lane & 3) * 8;
#pragma unroll
    for (int t = 0; t < 2 * M; ++t) {
      const int i = 8 * (t & 1);
      const floatx16_t& x = p[t >> 1];
      const uint4 pb = make_uint4(pack2<DT>(x[i], x[i + 1]), pack2<DT>(x[i + 2], x[i + 3]), pack2<DT>(x[i + 4], x[i + 5]),
                                  pack2<DT>(x[i + 6], x[i + 7]));
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) {
        const lds_char* const at = vr + t * 16 * kRowBytes + (((2 * ct + g1) ^ (2 * r4 + h)) << 5);
        const uint2 v0 = lds_read_transposed(at), v1 = lds_read_transposed(at + 8 * kRowBytes);
        o[ct] = mfma_32x32x16<DT>(make_uint4(v0.x, v0.y, v1.x, v1.y), pb, o[ct]);
      }
    }
  }
};

template <int DT>
__device__ __forceinline__ void store_channels(char* out_row, int ct, int h, const floatx16_t& o, float inv) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<uint2*>(out_row + ct * 64 + i * 16 + h * 8) =
        make_uint2(pack2<DT>(o[4 * i] * inv, o[4 * i + 1] * inv), pack2<DT>(o[4 * i + 2] * inv, o[4 * i + 3] * inv));
}

// The lane's number anew: what is only needed after a loop need not live in registers through it.
__device__ __forceinline__ int lane_again() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
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
    const int tok = row / a.n_rep, qh = head * a.n_rep + row - tok * a.n_rep;
    lim = min(sp.first + tok + 1, a.kv_cap);
    q = a.q + (size_t)(sp.lo + tok) * a.q_stride + qh * kRowBytes;
    out = a.out + ((size_t)(sp.lo + tok) * a.n_q_heads + qh) * kRowBytes;
  }
};

// ---- partial results of a part of the K / V rows ------------------------------------------------------------------------------
// Per 32 query rows: o as the lanes hold it (four channel tiles of 16 floats a lane), then m and l of every lane.  Written through
// to memory and read past the caches: another workgroup of the launch reads them (see arrive_add).  Only lanes whose row is
// there take part.
constexpr int kPartFloats = 32 * kD + 2 * 64;
__device__ __forceinline__ void store_partial(float* slot, int ct, const floatx16_t& o, int lane) {
  unsigned long long* const p = reinterpret_cast<unsigned long long*>(slot + ct * 1024) + lane;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    store_coherent(p + i * 64, (unsigned long long)__float_as_uint(o[2 * i]) | (unsigned long long)__float_as_uint(o[2 * i + 1]) << 32);
}
__device__ __forceinline__ void store_partial_sums(float* slot, float m, float l, int lane) {
  store_coherent(reinterpret_cast<unsigned long long*>(slot + 32 * kD) + lane,
                 (unsigned long long)__float_as_uint(m) | (unsigned long long)__float_as_uint(l) << 32);
}
// Channel tiles ct0 .. ct0 + CT - 1 of n slots, `pitch` floats apart, joined; BATCH slots' loads are under way together.
template <int CT, int BATCH>
__device__ __forceinline__ void join_partials(const float* slots, size_t pitch, int n, int ct0, int lane, floatx16_t (&o)[CT],
                                              float& l) {
  float m = -FLT_MAX;
  l = 0.f;
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = floatx16_t{0.f};
  for (int p0 = 0; p0 < n; p0 += BATCH) {
    unsigned long long ml[BATCH], w[BATCH][CT][8];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const float* const slot = slots + (size_t)min(p0 + k, n - 1) * pitch;
      ml[k] = load_coherent(reinterpret_cast<const unsigned long long*>(slot + 32 * kD) + lane);
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          w[k][c][i] = load_coherent(reinterpret_cast<const unsigned long long*>(slot + (ct0 + c) * 1024) + i * 64 + lane);
    }
    float to = m;
#pragma unroll
    for (int k = 0; k < BATCH; ++k) to = fmaxf(to, __uint_as_float((uint32_t)ml[k]));
    const float alpha = __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= alpha;
#pragma unroll
    for (int c = 0; c < CT; ++c) o[c] *= alpha;
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const float f = p0 + k < n ? __builtin_amdgcn_exp2f(__uint_as_float((uint32_t)ml[k]) - m) : 0.f;
      l += f * __uint_as_float((uint32_t)(ml[k] >> 32));
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          o[c][2 * i] += f * __uint_as_float((uint32_t)w[k][c][i]);
          o[c][2 * i + 1] += f * __uint_as_float((uint32_t)(w[k][c][i] >> 32));
        }
    }
  }
}

constexpr int kSideTile = 32;    // rows of K and V per wavefront and step where the wavefronts go side by side
constexpr int kSideWaves = 3;    // of four: three such workgroups fit a CU's LDS
constexpr int kSideStep = kSideWaves * kSideTile;
#ifndef MAXP
#define MAXP 48
#endif
constexpr int kMostParts = MAXP;  // of a tile
constexpr int kSideLeast = 2;    // steps of a part there, at least
constexpr int kSharedLeast = 8;  // steps of 64 rows of a part where the wavefronts share the tiles, at least

// ---- which workgroup does what -----------------------------------------------------------------------------------------------
// A sequence's query rows per kv head are cut into tiles of 128; the last one, where it has at most 32, goes through its K / V
// rows side by side, the others share them.  Where there are partial results to hand on (a cache's workspace), the K / V rows of
// a tile are split into parts of `step` steps, one length for all sequences of the call, so that unequal ones keep the GPU busy to
// the end: `step` is the call's steps over the number of parts wanted.  Lengths lie on the GPU, so every workgroup works
// this out for itself, one sequence a lane.
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
  __device__ __forceinline__ int parts(int step) const {  // that its tiles have at most; more tiles than counters: not split
    const int n = steps<SIDE>();
    return n <= step || (!SIDE && tiles >= kSelBins - 1) ? 1 : min((n + step - 1) / step, kMostParts);
  }
  template <bool SIDE>
  __device__ __forceinline__ int items(int step) const {
    return SIDE ? (aside ? parts<true>(step) : 0) : tiles * parts<false>(step);
  }
};
struct Item {
  PromptSpan sp;
  int b, at;    // sequence; which of its items
  int parts;    // of its tiles
  int step;     // steps of a part
  int slot;     // partial results: the place of the sequence's first item
};
// Sum of the lanes' values, the same in every lane and workgroup.
__device__ __forceinline__ float wave_sum_ordered(float x) {
  x += row_ror<8>(x), x += row_ror<4>(x), x += row_ror<2>(x), x += row_ror<1>(x);
  const int v = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(v, 0)) + __int_as_float(__builtin_amdgcn_readlane(v, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(v, 32)) + __int_as_float(__builtin_amdgcn_readlane(v, 48)));
}
// Item number j of the launch's (per kv head); false: there are fewer.
template <bool SIDE>
__device__ __forceinline__ bool find_item(const PromptArgs& a, int j, int lane, Item& it) {
  const int wanted = SIDE ? a.side_parts : a.shared_parts;  // 0: nothing is split
  it.step = 1 << 30;
  if (wanted) {
    float all = 0.f;
    int64_t tokens = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      const SequenceWork w(a, b0 + lane, lane, tokens);
      all += wave_sum_ordered((float)(SIDE ? (w.aside ? 1 : 0) : w.tiles) * (float)w.steps<SIDE>());
    }
    it.step = max(SIDE ? kSideLeast : kSharedLeast, (int)ceilf(all / (float)wanted));
    it.step = __builtin_amdgcn_readfirstlane(it.step);
  }
  int before = 0, slots = 0;
  int64_t tokens = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const SequenceWork w(a, b0 + lane, lane, tokens);
    const int parts = w.parts<SIDE>(it.step), n = w.items<SIDE>(it.step), split = parts > 1 ? n : 0;
    const int upto = before + (int)wave_incl_scan_u32((uint32_t)n, lane);
    const int slots_upto = slots + (int)wave_incl_scan_u32((uint32_t)split, lane);
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
  }
  return false;
}


// The wavefronts' results of a side-by-side tile: each puts its own into its LDS, then takes one channel tile of all.
template <int DT>
__device__ __forceinline__ void join_side_by_side(const PromptArgs& a, const Item& it, int head, const Rows32<DT>& st, int wave,
                                                  lds_char* lds, uint32_t* flag) {
  const int lane = lane_again(), h = lane >> 5;
  const int unit = it.b * a.n_kv_heads + head, n_rows = it.sp.n * a.n_rep, part = it.at, n_parts = it.parts;
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
  floatx16_t o[1] = {floatx16_t{0.f}};
#pragma unroll
  for (int w = 0; w < kSideWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(of[w].x - m);
    sum += f * of[w].y;
    const lds_float* const p = (const lds_float*)(lds + w * 2 * kSideTile * kRowBytes);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[0][i] += f * p[(wave * 16 + i) * 64 + lane];
  }
  if (n_parts > 1) {
    float* const slots = a.side_partials + ((size_t)head * a.side_slots + it.slot) * kPartFloats;
    if (row.there) {
      store_partial(slots + (size_t)part * kPartFloats, wave, o[0], lane);
      if (wave == 0) store_partial_sums(slots + (size_t)part * kPartFloats, m, sum, lane);
    }
    uint32_t* const counter = a.counters + (size_t)unit * kSelBins;
    if (arrive_add(counter, 1u, flag, wave == 0 && lane == 0) != (uint32_t)n_parts - 1) return;  // not the last one
    if (row.there) join_partials<1, 8>(slots, kPartFloats, n_parts, wave, lane, o, sum);
    if (wave == 0 && lane == 0) store_coherent(counter, 0u);
  }
  if (row.there) store_channels<DT>(row.out, wave, h, o[0], sum > 0.f ? 1.f / sum : 0.f);
}

// Up to 32 query rows: all four wavefronts hold them and go side by side through the K / V rows, each through 32 of every 128,
// in 16 KiB of LDS of its own, so that nobody waits for anybody.  The next K rows are loaded once this step's logits are
// there, the next V rows after its product.  Bound by memory.
template <int DT>
__device__ __forceinline__ void attend_side_by_side(const PromptArgs& a, const Item& it, int head, lds_char* lds, uint32_t* flag) {
  const PromptSpan sp = it.sp;
  const int unit = it.b * a.n_kv_heads + head, n_rows = sp.n * a.n_rep, row0 = n_rows / kRowTile * kRowTile;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int n_kv = min(sp.first + (n_rows - 1) / a.n_rep + 1, a.kv_cap);
  const int all = (n_kv + kSideStep - 1) / kSideStep, n_parts = it.parts;
  const int begin = (int)((int64_t)all * it.at / n_parts), end = (int)((int64_t)all * (it.at + 1) / n_parts);
  const QueryRow row(a, sp, head, row0 + n, n_rows);
  const int least = __builtin_amdgcn_readfirstlane(row.lim);  // the first row's
  const UnitRows rows(a, unit, head, sp.lo);
  lds_char* const kt = lds + wave * 2 * kSideTile * kRowBytes;
  lds_char* const vt = kt + kSideTile * kRowBytes;
  const RowLoads<false, 8, 1> kl(0, lane, rows.k_stride);
  const RowLoads<true, 8, 1> vl(0, lane, rows.v_stride);
  int t0 = begin * kSideStep + wave * kSideTile;
  const int stop = wave < kSideWaves ? min(end * kSideStep, n_kv) : 0;
  int block = 0;
  if (t0 < stop) {
    const size_t r = rows.row(rows.block_of(t0), t0);
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - t0, kt, 0, lane);
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - t0, vt, 0, lane);
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
    floatx16_t s[1];
    wait_loads<8>();
    Rows32<DT>::scores(kt, q, n, h, s);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - next, kt, 0, lane);
    block = rows.block_of(next + kSideStep < stop ? next + kSideStep : next);  // for the step after the next: the list is far away
    st.weights(s, a.scale, t0 + kSideTile > least, row.lim - t0, h);
    wait_loads<8>();
    st.add_values(vt, s, lane, h);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - next, vt, 0, lane);
  }
  wait_loads<0>();
  join_side_by_side<DT>(a, it, head, st, wave, lds, flag);
}
// The results of a tile of shared rows, through partial results where its K / V rows were split.
template <int DT>
__device__ __forceinline__ void finish_shared(const PromptArgs& a, const Item& it, int head, int tile, int turned, int part, int n_parts,
                                              Rows32<DT>& st, int wave, uint32_t* flag) {
  const int lane = lane_again(), h = lane >> 5;
  const int unit = it.b * a.n_kv_heads + head;
  const QueryRow row(a, it.sp, head, tile * kRowTile + wave * 32 + (lane & 31), it.sp.n * a.n_rep);
  float l = halves_sum(st.l);
  if (n_parts > 1) {
    float* const slots = a.shared_partials + (((size_t)head * a.shared_slots + it.slot + turned * it.parts) * 4 + wave) * kPartFloats;
    if (row.there) {
      float* const slot = slots + (size_t)part * 4 * kPartFloats;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) store_partial(slot, ct, st.o[ct], lane);
      store_partial_sums(slot, st.m, l, lane);
    }
    uint32_t* const counter = a.counters + (size_t)unit * kSelBins + 1 + tile;
    if (arrive_add(counter, 1u, flag, wave == 0 && lane == 0) != (uint32_t)n_parts - 1) return;  // not the last one
    if (row.there) join_partials<4, 2>(slots, 4 * kPartFloats, n_parts, 0, lane, st.o, l);
    if (wave == 0 && lane == 0) store_coherent(counter, 0u);
  }
  if (!row.there) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) store_channels<DT>(row.out, ct, h, st.o[ct], inv);
}

// 128 query rows, 32 a wavefront; the K / V rows go through LDS 64 at a time, two tiles of each, shared by the wavefronts.
template <int DT>
__device__ __forceinline__ void attend_shared(const PromptArgs& a, const Item& it, int head, lds_char* lds, uint32_t* flag) {
  const PromptSpan sp = it.sp;
  const int unit = it.b * a.n_kv_heads + head, n_rows = sp.n * a.n_rep;
  const int tiles = n_rows / kRowTile + (n_rows % kRowTile > kSideRows ? 1 : 0);
  // the tiles that attend over the most rows first
  const int turned = it.at / it.parts, tile = tiles - 1 - turned, part = it.at - turned * it.parts;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int row0 = tile * kRowTile;
  const int n_kv = min(sp.first + (min(row0 + kRowTile, n_rows) - 1) / a.n_rep + 1, a.kv_cap);
  const int all = (n_kv + kTile - 1) / kTile, n_parts = min(it.parts, (all + it.step - 1) / it.step);
  if (part >= n_parts) return;  // the first tiles of a prompt attend over fewer rows than the last one
  const int begin = (int)((int64_t)all * part / n_parts), end = (int)((int64_t)all * (part + 1) / n_parts);
  const QueryRow row(a, sp, head, row0 + wave * 32 + n, n_rows);
  const int least = __builtin_amdgcn_readfirstlane(row.lim), most = __builtin_amdgcn_readlane(row.lim, 31);
  const UnitRows rows(a, unit, head, sp.lo);
  constexpr int kBytes = kTile * kRowBytes;
  const RowLoads<false, 4, 4> kl(wave, lane, rows.k_stride);
  const RowLoads<true, 4, 4> vl(wave, lane, rows.v_stride);
  const size_t r0 = rows.row(rows.block_of(begin * kTile), begin * kTile);
  kl.load(rows.k + r0 * rows.k_stride, rows.k_stride, n_kv - begin * kTile, lds, wave, lane);
  size_t r = r0;
  int block = rows.block_of(min(begin + 1, end - 1) * kTile);
  uint4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = a.load_q(row.q + s * 32 + h * 16);
  Rows32<DT> st;
  st.init();
  lds_char* const vt = lds + 2 * kBytes;
  for (int i = begin; i < end; ++i) {
    const int t0 = i * kTile, next = i + 1 < end ? t0 + kTile : t0, cur = (i - begin) & 1;
    const lds_char* const kt = lds + cur * kBytes;
    wait_loads<0>();
    meet();
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - t0, vt, wave, lane);
    r = rows.row(block, next);
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - next, lds + (cur ^ 1) * kBytes, wave, lane);
    block = rows.block_of(min(i + 2, end - 1) * kTile);
    floatx16_t s[1];
    if (t0 < most) {  // some of the wavefront's rows go that far
      Rows32<DT>::scores(kt, q, n, h, s);
      st.weights(s, a.scale, t0 + 32 > least, row.lim - t0, h);
    }
    wait_loads<4>();
    meet();
    if (t0 < most) st.add_values(vt, s, lane, h);
    if (t0 + 32 < most) {
      Rows32<DT>::scores(kt + 32 * kRowBytes, q, n, h, s);
      st.weights(s, a.scale, t0 + kTile > least, row.lim - t0 - 32, h);
      st.add_values(vt + 32 * kRowBytes, s, lane, h);
    }
  }
  wait_loads<0>();
  finish_shared<DT>(a, it, head, tile, turned, part, n_parts, st, wave, flag);
}

// The grid lists the side-by-side items first, then the shared ones, the kv heads of an item next to each other: with a multiple
// of 8 of them a head's K and V stay in one XCD's L2.  What has no work leaves at once.  A tile whose K / V rows are split hands
// its partial results to the last of its workgroups.
template <int DT>
__global__ __launch_bounds__(256, 3) void prompt_attn_kernel(PromptArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[3 * kTile * kRowBytes + kSideWaves * 64 * 8];
  __shared__ uint32_t flag;
  const int lane = threadIdx.x & 63;
  const bool side = blockIdx.x < (unsigned)a.side_grid;
  const unsigned id = side ? blockIdx.x : blockIdx.x - (unsigned)a.side_grid;
  const int j = (int)(id / (unsigned)a.n_kv_heads), head = (int)(id - (unsigned)j * (unsigned)a.n_kv_heads);
  Item it;
  if (side) {
    if (find_item<true>(a, j, lane, it)) attend_side_by_side<DT>(a, it, head, (lds_char*)lds, &flag);
  } else {
    if (find_item<false>(a, j, lane, it)) attend_shared<DT>(a, it, head, (lds_char*)lds, &flag);
  }
}

#ifndef SIDE_T
#define SIDE_T 1536
#endif
#ifndef SHARED_T
#define SHARED_T 768
#endif
// How the launch is cut.
PromptSplit prompt_split(int batch, int n_kv_heads, int n_rep, int n_tokens, int max_new, bool split) {
  PromptSplit sp = {};
  const int64_t rows = (int64_t)max_new * n_rep, all_rows = (int64_t)n_tokens * n_rep;
  const bool shared = rows > kSideRows;  // some sequence may have more rows than go side by side
  const int64_t seqs = std::min(batch, n_tokens);
  sp.side_parts = split ? std::max(1, SIDE_T / n_kv_heads) : 0;
  sp.shared_parts = split && shared ? std::max(1, SHARED_T / n_kv_heads) : 0;
  sp.side_grid = (seqs + sp.side_parts) * n_kv_heads;
  sp.shared_grid = shared ? (all_rows / kRowTile + seqs + sp.shared_parts) * n_kv_heads : 0;
  // Items of tiles in more than one part: at most twice the parts wanted, since ceil(x) < 2 x for x > 1.
  sp.side_slots = 2 * sp.side_parts;
  sp.shared_slots = 2 * sp.shared_parts;
  sp.side_floats = (size_t)sp.side_slots * n_kv_heads * kPartFloats;
  sp.shared_floats = (size_t)sp.shared_slots * n_kv_heads * 4 * kPartFloats;
  return sp;
}

// FIER_ESHAPE where the grid would not fit 32 bits, else FIER_OK or FIER_EHIP.
int launch_prompt_attn(int dtype, PromptArgs a, const PromptSplit& sp, hipStream_t st) {
  const int64_t grid = sp.side_grid + sp.shared_grid;
  if (a.max_new == 0) return FIER_OK;
  if (grid > INT32_MAX) return FIER_ESHAPE;
  a.side_grid = (int)sp.side_grid;
  a.side_parts = sp.side_parts, a.shared_parts = sp.shared_parts;
  a.side_slots = sp.side_slots, a.shared_slots = sp.shared_slots;
  a.shared_partials = a.side_partials + sp.side_floats;
  if (dtype == DT_F16)
    prompt_attn_kernel<DT_F16><<<(unsigned)grid, 256, 0, st>>>(a);
  else
    prompt_attn_kernel<DT_BF16><<<(unsigned)grid, 256, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? FIER_OK : FIER_EHIP;
}

}  // namespace fier
