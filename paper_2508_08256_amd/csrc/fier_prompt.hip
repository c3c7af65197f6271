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

// The N instructions of a wavefront that bring its share of a tile: rows 4 (N0 + STEP j) .. + 3.
template <bool V, int N, int STEP>
struct RowLoads {
  uint32_t chunk[N];  // offset of the lane's 16 bytes in its row; repeats where the permutation does
  int row[N];
  __device__ __forceinline__ RowLoads(int n0, int lane) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      row[j] = 4 * (n0 + STEP * j) + (lane >> 4);
      const int c = lane & 15;
      chunk[j] = 16u * (uint32_t)(V ? c ^ (((row[j] & 3) << 2) | ((row[j] >> 1) & 2)) : c ^ (row[j] & 15));
    }
  }
  // rows: how many the tile has; the others take the last one's (they get no weight)
  __device__ __forceinline__ void load(const char* src, int64_t stride, int rows, const lds_char* dst, int n0) const {
#pragma unroll
    for (int j = 0; j < N; ++j)
      load_rows_to_lds(src, (uint32_t)min(row[j], rows - 1) * (uint32_t)stride + chunk[j], dst + 4 * (n0 + STEP * j) * kRowBytes);
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

// The parts that n_tiles steps are split into, at most `most`, none shorter than `least` steps.
__device__ __forceinline__ int parts_of(int n_tiles, int most, int least) { return max(1, min(most, n_tiles / least)); }

constexpr int kSideTile = 32;    // rows of K and V per wavefront and step where the wavefronts go side by side
constexpr int kSideLeast = 2;    // steps of 128 rows of such a part, at least
constexpr int kSharedLeast = 8;  // steps of 64 rows of a part where the wavefronts share the tiles, at least

// Up to 32 query rows: all four wavefronts hold them and go side by side through the K / V rows, each through 32 of every 128,
// in 16 KiB of LDS of its own, so that nobody waits for anybody.  The next K rows are loaded once this step's logits are
// there, the next V rows after its product.  Bound by memory.
template <int DT>
__device__ __forceinline__ void attend_side_by_side(const PromptArgs& a, const PromptSpan& sp, int unit, int head, int row0,
                                                    int n_rows, int part, lds_char* lds, uint32_t* flag) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int n_kv = min(sp.first + (n_rows - 1) / a.n_rep + 1, a.kv_cap);
  const int all = (n_kv + 127) / 128, n_parts = parts_of(all, a.side_parts, kSideLeast);
  if (part >= n_parts) return;
  const int begin = (int)((int64_t)all * part / n_parts), end = (int)((int64_t)all * (part + 1) / n_parts);
  const QueryRow row(a, sp, head, row0 + n, n_rows);
  const int least = __builtin_amdgcn_readfirstlane(row.lim);  // the first row's
  const UnitRows rows(a, unit, head, sp.lo);
  lds_char* const kt = lds + wave * 2 * kSideTile * kRowBytes;
  lds_char* const vt = kt + kSideTile * kRowBytes;
  const RowLoads<false, 8, 1> kl(0, lane);
  const RowLoads<true, 8, 1> vl(0, lane);
  int t0 = begin * 128 + wave * kSideTile;
  const int stop = min(end * 128, n_kv);
  int block = 0;
  if (t0 < stop) {
    const size_t r = rows.row(rows.block_of(t0), t0);
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - t0, kt, 0);
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - t0, vt, 0);
    block = rows.block_of(t0 + 128 < stop ? t0 + 128 : t0);
  }
  uint4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = a.load_q(row.q + s * 32 + h * 16);
  Rows32<DT> st;
  st.init();
  for (; t0 < stop; t0 += 128) {
    const int next = t0 + 128 < stop ? t0 + 128 : t0;  // the last step loads its own rows once more
    const size_t r = rows.row(block, next);
    floatx16_t s[1];
    wait_loads<8>();
    Rows32<DT>::scores(kt, q, n, h, s);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - next, kt, 0);
    block = rows.block_of(next + 128 < stop ? next + 128 : next);  // for the step after the next: the list is far away
    st.weights(s, a.scale, t0 + kSideTile > least, row.lim - t0, h);
    wait_loads<8>();
    st.add_values(vt, s, lane, h);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - next, vt, 0);
  }
  wait_loads<0>();
  // the four wavefronts' results: each puts its own into its LDS, then takes one channel tile of all
  const float l = halves_sum(st.l);
  __attribute__((address_space(3))) float* const mine = (__attribute__((address_space(3))) float*)kt;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) mine[(ct * 16 + i) * 64 + lane] = st.o[ct][i];
  __attribute__((address_space(3))) float2* const ml = (__attribute__((address_space(3))) float2*)(lds + 8 * kSideTile * kRowBytes);
  typedef float f2_t __attribute__((ext_vector_type(2)));
  *(__attribute__((address_space(3))) f2_t*)&ml[wave * 64 + lane] = f2_t{st.m, l};
  meet();
  float m = -FLT_MAX, sum = 0.f;
  f2_t of[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    of[w] = *(__attribute__((address_space(3))) f2_t*)&ml[w * 64 + lane];
    m = fmaxf(m, of[w].x);
  }
  floatx16_t o[1] = {floatx16_t{0.f}};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(of[w].x - m);
    sum += f * of[w].y;
    const __attribute__((address_space(3))) float* const p = (const __attribute__((address_space(3))) float*)(lds + w * 2 * kSideTile * kRowBytes);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[0][i] += f * p[(wave * 16 + i) * 64 + lane];
  }
  if (n_parts > 1) {
    float* const slots = a.side_partials + (size_t)unit * a.side_parts * kPartFloats;
    if (row.there) {
      store_partial(slots + (size_t)part * kPartFloats, wave, o[0], lane);
      if (wave == 0) store_partial_sums(slots + (size_t)part * kPartFloats, m, sum, lane);
    }
    uint32_t* const counter = a.counters + (size_t)unit * kSelBins;
    if (!last_arriver(counter, (uint32_t)n_parts, flag)) return;
    if (row.there) join_partials<1, 8>(slots, kPartFloats, n_parts, wave, lane, o, sum);
    if (threadIdx.x == 0) store_coherent(counter, 0u);
  }
  if (row.there) store_channels<DT>(row.out, wave, h, o[0], sum > 0.f ? 1.f / sum : 0.f);
}

// 128 query rows, 32 a wavefront; the K / V rows go through LDS 64 at a time, two tiles of each, shared by the wavefronts.
template <int DT>
__device__ __forceinline__ void attend_shared(const PromptArgs& a, const PromptSpan& sp, int unit, int head, int tile,
                                              int n_rows, int part, lds_char* lds, uint32_t* flag) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int row0 = tile * kRowTile;
  const int n_kv = min(sp.first + (min(row0 + kRowTile, n_rows) - 1) / a.n_rep + 1, a.kv_cap);
  const int all = (n_kv + kTile - 1) / kTile, n_parts = parts_of(all, a.shared_parts, kSharedLeast);
  if (part >= n_parts) return;
  const int begin = (int)((int64_t)all * part / n_parts), end = (int)((int64_t)all * (part + 1) / n_parts);
  const QueryRow row(a, sp, head, row0 + wave * 32 + n, n_rows);
  const int least = __builtin_amdgcn_readfirstlane(row.lim), most = __builtin_amdgcn_readlane(row.lim, 31);
  const UnitRows rows(a, unit, head, sp.lo);
  constexpr int kBytes = kTile * kRowBytes;
  const RowLoads<false, 4, 4> kl(wave, lane);
  const RowLoads<true, 4, 4> vl(wave, lane);
  const size_t r0 = rows.row(rows.block_of(begin * kTile), begin * kTile);
  kl.load(rows.k + r0 * rows.k_stride, rows.k_stride, n_kv - begin * kTile, lds, wave);
  vl.load(rows.v + r0 * rows.v_stride, rows.v_stride, n_kv - begin * kTile, lds + 2 * kBytes, wave);
  int block = rows.block_of(min(begin + 1, end - 1) * kTile);
  uint4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = a.load_q(row.q + s * 32 + h * 16);
  Rows32<DT> st;
  st.init();
  for (int i = begin; i < end; ++i) {
    const int t0 = i * kTile, next = i + 1 < end ? t0 + kTile : t0, cur = (i - begin) & 1;
    lds_char* const kt = lds + cur * kBytes;
    lds_char* const vt = lds + (2 + cur) * kBytes;
    const size_t r = rows.row(block, next);
    const bool needed = t0 < most;  // none of the wavefront's rows goes that far
    floatx16_t s[2];
    wait_loads<4>();
    meet();
    kl.load(rows.k + r * rows.k_stride, rows.k_stride, n_kv - next, lds + (cur ^ 1) * kBytes, wave);
    block = rows.block_of(min(i + 2, end - 1) * kTile);
    if (needed) {
      Rows32<DT>::scores(kt, q, n, h, s);
      st.weights(s, a.scale, t0 + kTile > least, row.lim - t0, h);
    }
    wait_loads<4>();
    meet();
    vl.load(rows.v + r * rows.v_stride, rows.v_stride, n_kv - next, lds + (2 + (cur ^ 1)) * kBytes, wave);
    if (needed) st.add_values(vt, s, lane, h);
  }
  wait_loads<0>();
  float l = halves_sum(st.l);
  if (n_parts > 1) {
    const size_t item = (size_t)unit * a.row_tiles + tile;
    float* const slots = a.shared_partials + (item * a.shared_parts * 4 + wave) * kPartFloats;
    if (row.there) {
      float* const slot = slots + (size_t)part * 4 * kPartFloats;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) store_partial(slot, ct, st.o[ct], lane);
      store_partial_sums(slot, st.m, l, lane);
    }
    uint32_t* const counter = a.counters + (size_t)unit * kSelBins + 1 + tile;
    if (!last_arriver(counter, (uint32_t)n_parts, flag)) return;
    if (row.there) join_partials<4, 2>(slots, 4 * kPartFloats, n_parts, 0, lane, st.o, l);
    if (threadIdx.x == 0) store_coherent(counter, 0u);
  }
  if (!row.there) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) store_channels<DT>(row.out, ct, h, st.o[ct], inv);
}

// The query rows of a unit are cut into tiles of 128; the last one, where it has at most 32, goes through its K / V rows side by
// side.  The grid lists a place for that one of every unit first, side_parts times, then the whole tiles, the last ones (which
// attend over the most rows) first; units fastest, so that with a multiple of 8 units a unit's K and V stay in one XCD's L2.
// What has no work leaves at once.  A tile whose K / V rows are split hands its partial results to the last of its workgroups.
template <int DT>
__global__ __launch_bounds__(256, 2) void prompt_attn_kernel(PromptArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile * kRowBytes + 4 * 64 * 8];
  __shared__ uint32_t flag;
  const unsigned id = blockIdx.x, side = (unsigned)a.units * (unsigned)a.side_parts;
  const unsigned place = (id < side ? id : id - side) / (unsigned)a.units;
  const int unit = (int)((id < side ? id : id - side) - place * (unsigned)a.units);
  const int b = unit / a.n_kv_heads, head = unit - b * a.n_kv_heads;
  PromptSpan sp = a.span(b);
  sp = {__builtin_amdgcn_readfirstlane(sp.lo), __builtin_amdgcn_readfirstlane(sp.n), __builtin_amdgcn_readfirstlane(sp.first)};
  const int n_rows = sp.n * a.n_rep, whole = n_rows / kRowTile, rest = n_rows - whole * kRowTile;
  const bool aside = rest > 0 && rest <= kSideRows;
  if (id < side) {
    if (aside) attend_side_by_side<DT>(a, sp, unit, head, whole * kRowTile, n_rows, (int)place, (lds_char*)lds, &flag);
    return;
  }
  const int tile = a.row_tiles - 1 - (int)(place / (unsigned)a.shared_parts);
  if (tile < whole || (tile == whole && rest > kSideRows))
    attend_shared<DT>(a, sp, unit, head, tile, n_rows, (int)(place % (unsigned)a.shared_parts), (lds_char*)lds, &flag);
}

// How many parts the K / V rows are split into, and the workspace for them.
PromptSplit prompt_split(int units, int n_rep, int max_new, int kv_cap) {
  PromptSplit sp;
  const int64_t rows = (int64_t)max_new * n_rep;
  sp.row_tiles = (int)((rows + kRowTile - 1) / kRowTile);
  if (rows <= kSideRows) sp.row_tiles = 0;  // every unit's rows go side by side
  const int64_t tiles = (int64_t)units * sp.row_tiles;
  sp.side_parts = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(2048 / units, 64), kv_cap / (128 * kSideLeast)));
  sp.shared_parts = tiles == 0 || sp.row_tiles >= kSelBins - 1
                        ? 1
                        : (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, kv_cap / (kTile * kSharedLeast)));
  sp.side_floats = sp.side_parts > 1 ? (size_t)units * sp.side_parts * kPartFloats : 0;
  sp.shared_floats = sp.shared_parts > 1 ? (size_t)tiles * sp.shared_parts * 4 * kPartFloats : 0;
  return sp;
}

// FIER_ESHAPE where the grid would not fit 32 bits, else FIER_OK or FIER_EHIP.
int launch_prompt_attn(int dtype, const PromptArgs& a, hipStream_t st) {
  const int64_t grid = (int64_t)a.units * a.side_parts + (int64_t)a.units * a.row_tiles * a.shared_parts;
  if (a.max_new == 0) return FIER_OK;
  if (grid > INT32_MAX) return FIER_ESHAPE;
  if (dtype == DT_F16)
    prompt_attn_kernel<DT_F16><<<(unsigned)grid, 256, 0, st>>>(a);
  else
    prompt_attn_kernel<DT_BF16><<<(unsigned)grid, 256, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? FIER_OK : FIER_EHIP;
}

}  // namespace fier
