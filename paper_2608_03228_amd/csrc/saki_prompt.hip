// Causal attention of whole prompts for gfx950 (CDNA4, wave64):
//
//   prompt_attend_kernel      bf16
//   prompt_split_kernel       float32 keys and values as pairs of fp16 parts
//   prompt_attend_f32_kernel  float32 on those parts

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "saki.h"
#include "saki_internal.h"
#include "saki_topk.h"

namespace {

using saki::kHeadDim;
using saki_dev::kWave;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kScale = 0.08838834764831845f;  // 1 / sqrt(d)
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kRows = 128;    // query rows of a work-group (32 a wave)
constexpr int kKeys = 64;     // keys of a tile
// A row's sums are scaled down only once a score passes the maximum they go by
// by this many powers of two: a weight may be 2^kSlack, which neither bf16 nor
// the sums mind, and most tiles that bring a new maximum to one of a wave's 32
// rows cost no pass over its sums.
constexpr float kSlack = 8.f;

struct PromptArgs {
  const void *q, *k, *v;
  size_t ld_q, ld_k, ld_v;  // elements between tokens
  const int* cu;
  int B, H_q, H_kv, T;
  void* out;
  int tiles;  // row blocks of all prompts, at most
};

// Block `x` of `rows` rows of the packed prompts.  The rows of one KV head are
// (token, one of its G query heads) pairs, token after token; a prompt's blocks
// start at floor(first row / rows) + b, which leaves each prompt its own ones
// (with gaps), so that a block finds its prompt by a search of the offsets.
struct Block {
  int b, start, len, row0;  // prompt, its first token and length, first row in it; len = 0: none
};
__device__ __forceinline__ Block find_block(const PromptArgs& a, int x, int G, int rows) {
  auto at = [&](int b) { return min(max(a.cu[b], 0), a.T); };
  int lo = 0, n = a.B;  // the prompt is one of lo .. lo + n - 1: a wave tells 64 parts of them apart at once
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave, i = (int)(threadIdx.x % kWave) * step;
    const bool below = i < n && (long long)at(lo + i) * G / rows + lo + i <= x;
    const uint64_t which = __ballot(below);  // none: the block lies before the first prompt
    const int part = which ? (63 - __builtin_clzll(which)) * step : 0;
    n = min(n - part, step);
    lo += part;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  Block r;
  r.b = lo;
  r.start = at(lo);
  r.len = max(at(lo + 1) - r.start, 0);
  const long long row0 = (x - ((long long)r.start * G / rows + lo)) * rows;
  if (row0 < 0 || row0 >= (long long)r.len * G) r.len = 0;
  r.row0 = (int)row0;
  return r;
}

__device__ __forceinline__ float swap32(float v) {
  return __uint_as_float(saki_dev::xor_shfl_u32(__float_as_uint(v), 32));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  bf16x2_t v = {(__bf16)a, (__bf16)b};
  uint32_t r;
  __builtin_memcpy(&r, &v, sizeof(r));
  return r;
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// Adds a value's elements that are not finite to a lane's sums.
template <typename T>
__device__ __forceinline__ void add_odd(const T* v, f32x16_t* o) {
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = (float)v[32 * d + 8 * (i / 4) + i % 4];
      if (!finite(x)) o[d][i] += x;
    }
}

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// out_t = sum_u p_u v_u over the keys u <= t of a prompt.  A work-group takes 128
// rows (32 a wave) and reads the keys and values up to its last token in tiles
// of 64, staged into LDS by direct loads a tile ahead; 64 KB a group, two groups
// a CU, whose waves fill each other's pauses.  S^T = K Q^T leaves a lane with
// scores of one row (half of a tile's keys; lane + 32 has the others), so the
// softmax is in registers but for one exchange, and its weights, rounded to
// bf16, are at once the operand of O^T = V^T P^T, whose other operand the
// transposing LDS reads form.  (A weight's rounding, 2^-8 of it, is what one
// product in place of two costs: error 0.0019-0.0022 of the output, 0.0016 of
// which is the output's own rounding.)  Key pieces are staged rotated by their
// row, so that neither read meets bank conflicts (0 counted).  A prompt's blocks
// with most keys come first in the launch; of several prompts the last one's do.
// KS = 2: 64 rows, and two waves share a row's keys, 32 of each tile; their
// sums meet at the end (see halves_better).
// Bound by power and the MFMA: 0.95-1.06 PFLOP/s at 8,192 tokens of 32 / 8
// heads depending on the card (a large bf16 matrix product reaches 1.15), the
// MFMA 55% busy at a clock of 1.8 GHz.  Raising the waves' priority around the
// products or the softmax changed nothing.
template <int KS>
__global__ __launch_bounds__(256, 2) void prompt_attend_kernel(PromptArgs a) {
  constexpr int kBlockRows = kRows / KS;
  // two arrays, and the loop below unrolled over them: a read of one is then
  // known not to meet the loads into the other, and does not wait for them
  constexpr int kTileBytes = kKeys * kHeadDim * 2;
  __shared__ alignas(1024) uint8_t lds_a[2 * kTileBytes], lds_b[2 * kTileBytes];  // keys, values
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int hk = blockIdx.x % a.H_kv, G = a.H_q / a.H_kv;
  const Block blk = find_block(a, a.tiles - 1 - (int)(blockIdx.x / a.H_kv), G, kBlockRows);
  if (blk.len == 0) return;
  const int n_rows = (int)min((long long)blk.len * G - blk.row0, (long long)kBlockRows);
  const int n = lane % 32, h = lane / 32;

  // this wave's 32 rows and its part of a tile's keys; this lane's row, its token and head
  const int rw = KS == 1 ? wave * 32 : wave % 2 * 32, b0 = KS == 1 ? 0 : wave / 2;
  const int row = min(rw + n, n_rows - 1) + blk.row0;
  const int pos = row / G;
  const size_t q_at = (size_t)(blk.start + pos) * a.ld_q + (size_t)(hk * G + row % G) * kHeadDim;
  bf16x8_t q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const uint4 v = *reinterpret_cast<const uint4*>((const __bf16*)a.q + q_at + 16 * s + 8 * h);
    __builtin_memcpy(&q[s], &v, 16);
  }
  const int pos_lo = (blk.row0 + min(rw, n_rows - 1)) / G;
  const int pos_hi = (blk.row0 + min(rw + 31, n_rows - 1)) / G;
  const int n_tiles = (blk.row0 + n_rows - 1) / G / kKeys + 1;

  // staging: a wave's load takes 4 rows of 16 pieces; piece c of key row r goes
  // to place c ^ (r % 16) (keys), c ^ (r % 4 * 4) (values)
  const __bf16* kp = (const __bf16*)a.k + (size_t)blk.start * a.ld_k + (size_t)hk * kHeadDim;
  const __bf16* vp = (const __bf16*)a.v + (size_t)blk.start * a.ld_v + (size_t)hk * kHeadDim;
  uint32_t k_off[4], v_off[4];  // bytes from a tile's first key row; the same for every whole tile
  auto offsets = [&](int last) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = 16 * wave + 4 * u + lane / 16, at = min(r, last);
      k_off[u] = (uint32_t)at * (uint32_t)(2 * a.ld_k) + ((lane % 16) ^ (r % 16)) * 16;
      v_off[u] = (uint32_t)at * (uint32_t)(2 * a.ld_v) + ((lane % 16) ^ (r % 4 * 4)) * 16;
    }
  };
  auto stage = [&](int t, uint8_t* to) __attribute__((always_inline)) {
    if ((t + 1) * kKeys > blk.len) offsets(blk.len - 1 - t * kKeys);  // (the last tile: past the prompt, its last key)
    const uint8_t* kt = (const uint8_t*)(kp + (size_t)t * kKeys * a.ld_k);
    const uint8_t* vt = (const uint8_t*)(vp + (size_t)t * kKeys * a.ld_v);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      __builtin_amdgcn_global_load_lds((global_void*)(kt + k_off[u]), (lds_void*)(to + (16 * wave + 4 * u) * 256), 16,
                                       0, 0);
      __builtin_amdgcn_global_load_lds((global_void*)(vt + v_off[u]),
                                       (lds_void*)(to + kTileBytes + (16 * wave + 4 * u) * 256), 16, 0, 0);
    }
  };

  f32x16_t o[4];
  float m, l;
  const int k_lane = n * 256 + ((h ^ (lane % 16)) * 16);
  const int vs = lane % 16, vg = lane / 16;
  const int v_lane = (4 * (vg / 2) + vs / 4) * 256 + 32 * (vg % 2) + 8 * (vs % 4);

  // Elements of a tile's values that are not finite become zero, in LDS; returns
  // which of its keys have such ones.  (A work-group's threads take a quarter of a
  // row each; the callers' barriers stand between two tiles' uses of `odd`.)
  __shared__ uint32_t odd[4];
  auto clear_odd = [&](uint8_t* vt) {
    uint8_t* p = vt + threadIdx.x * 64;
    bool any = false;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint16_t x[8];
      __builtin_memcpy(x, p + 16 * u, 16);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((x[e] & 0x7f80) == 0x7f80) any = true, x[e] = 0;
      __builtin_memcpy(p + 16 * u, x, 16);
    }
    uint64_t which = __ballot(any);  // 16 rows of four lanes
    which |= which >> 1;
    which |= which >> 2;
    uint32_t rows = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r) rows |= (uint32_t)(which >> (4 * r) & 1) << r;
    if (lane == 0) odd[wave] = rows;
    __syncthreads();
    return (uint64_t)(odd[0] | odd[1] << 16) | (uint64_t)(odd[2] | odd[3] << 16) << 32;
  };

  auto tile = [&](int t, uint8_t* kt, uint8_t* next, auto careful) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's part of tile t
    __syncthreads();
    if (t + 1 < n_tiles) stage(t + 1, next);
    uint64_t odd_keys = 0;
    if constexpr (careful) odd_keys = clear_odd(kt + kTileBytes);
    if (t * kKeys > pos_hi) return;
    const uint8_t* vt = kt + kTileBytes;
    f32x16_t s[2 / KS];
#pragma unroll
    for (int b = 0; b < 2 / KS; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        bf16x8_t kf;
        __builtin_memcpy(&kf, kt + (b + b0) * 32 * 256 + (k_lane ^ (x * 32)), 16);
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[x], s[b], 0, 0, 0);
      }
    }
    if (t * kKeys + kKeys - 1 > pos_lo) {
#pragma unroll
      for (int b = 0; b < 2 / KS; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t * kKeys + 32 * (b + b0) + 8 * (i / 4) + 4 * h + i % 4 > pos) s[b][i] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 32 / KS; ++i) top = fmaxf(top, s[i / 16][i % 16]);
    top = fmaxf(top, swap32(top));
    if (__any(top > m + kSlack / (kScale * kLog2e))) {
      const float m1 = fmaxf(m, top);
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m1) * (kScale * kLog2e));
      m = m1;
      l *= keep;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= keep;
    }
    // (a part of the keys may hold none that a row sees)
    const float shift = KS > 1 && m == -INFINITY ? 0.f : -m * (kScale * kLog2e);
    uint32_t p[16 / KS];
#pragma unroll
    for (int b = 0; b < 2 / KS; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], kScale * kLog2e, shift));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], kScale * kLog2e, shift));
        l += p0 + p1;
        p[8 * b + i / 2] = pack_bf16(p0, p1);
      }
#pragma unroll
    for (int x = 0; x < 4 / KS; ++x) {  // 16 keys each
      bf16x8_t pf;
      __builtin_memcpy(&pf, &p[4 * x], 16);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
        const uint8_t* at = vt + (x + 2 * b0) * 16 * 256 + (v_lane ^ ((d ^ (vs / 4)) * 64));
        const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds_void*)at);
        const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds_void*)(at + 8 * 256));
        bf16x8_t vf;
        __builtin_memcpy(&vf, &lo, 8);
        __builtin_memcpy((char*)&vf + 8, &hi, 8);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[d], 0, 0, 0);
      }
    }
    if constexpr (careful) {
      if (KS == 2) odd_keys &= 0xffffffffull << 32 * b0;
      for (; odd_keys; odd_keys &= odd_keys - 1) {
        const int u = t * kKeys + __builtin_ctzll(odd_keys);
        if (u <= pos) add_odd(vp + (size_t)u * a.ld_v + 4 * h, o);
      }
    }
  };
  // A value that is not finite would reach rows that do not see its token, as 0
  // times it.  Where a sum of the group is not finite all is done again, such
  // elements taken out of the tiles and added to the rows that see them (0.2 us a
  // call where nothing is; one loop for both took 5% more in halved blocks).
  __shared__ bool again;
  if (threadIdx.x == 0) again = false;
  auto sums = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    m = -INFINITY, l = 0.f;
    offsets(kKeys - 1);
    stage(0, lds_a);
    for (int t = 0; t < n_tiles; t += 2) {
      tile(t, lds_a, lds_b, careful);
      if (t + 1 < n_tiles) tile(t + 1, lds_b, lds_a, careful);
    }
  };
  sums(std::false_type());
  float zero = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) zero = fmaf(o[d][i], 0.f, zero);
  if (zero != 0.f) again = true;
  __syncthreads();  // all tiles are read
  if (__builtin_expect(again, 0)) {
    sums(std::true_type());
    __syncthreads();
  }
  l += swap32(l);
  if constexpr (KS == 2) {  // the second waves' sums join the first ones', through the tiles' memory
    float* x = (float*)(rw ? lds_b : lds_a);  // [64 sums, maximum and weight][lane]
    static_assert(2 * kTileBytes >= 64 * kWave * 4);
    __shared__ float ml[2][2][kWave];
    if (b0 == 1) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(16 * d + i) * kWave + lane] = o[d][i];
      ml[rw / 32][0][lane] = m;
      ml[rw / 32][1][lane] = l;
    }
    __syncthreads();
    if (b0 == 1) return;
    const float m2 = ml[rw / 32][0][lane], l2 = ml[rw / 32][1][lane], m1 = fmaxf(m, m2);
    const float e1 = __builtin_amdgcn_exp2f((m - m1) * (kScale * kLog2e));
    const float e2 = __builtin_amdgcn_exp2f((m2 - m1) * (kScale * kLog2e));
    l = l * e1 + l2 * e2;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * e1 + x[(16 * d + i) * kWave + lane] * e2;
  }
  const float inv = 1.f / l;
  if (rw + n < n_rows) {
    __bf16* out = (__bf16*)a.out + ((size_t)(blk.start + pos) * a.H_q + hk * G + row % G) * kHeadDim;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<uint2*>(out + 32 * d + 2 * i + 4 * h) =
            make_uint2(pack_bf16(o[d][i] * inv, o[d][i + 1] * inv), pack_bf16(o[d][i + 2] * inv, o[d][i + 3] * inv));
  }
}

// float32 on the fp16 MFMA: x = (hi + lo) 2^-e with hi = fp16(x 2^e), lo = fp16(x
// 2^e - hi), where 2^e brings the largest element of a tile (of a query's row)
// to [2^14, 2^15).  What hi and lo leave is below 2^-22 |x|, or 2^-39 of that
// largest element, and a product is hi hi + lo hi + hi lo, all sums in float32:
// three fp16 products in place of one at an eighth of their rate.  A tile whose
// tokens' sizes are more than kSpread powers of two apart is `mixed`: there each
// token goes by its own power, so that none takes bits from another (seen or not).
// 4,096 tokens of 28 / 4 heads: 10.7 us for the split and 350-400 for the attention
// (310-340 TFLOP/s, the MFMA 63% busy); on the float32 MFMA it took 1,237 us.
// Every tile mixed: 414 us in all against 395; in halved blocks (5,000 tokens of
// 2 / 1 heads) 199 against 137, and 139 with the first one mixed.

constexpr int kSplitKeys = 32;
constexpr int kSplitTile = 4 * kSplitKeys * kHeadDim * 2;  // bytes: keys hi, lo, values hi, lo
constexpr int kSpread = 4;

// Exponents of a tile's keys and values (the least, of its largest elements),
// whether the tokens have their own, and the tokens whose values are not all finite.
struct TileExps {
  int k, v, mixed;
  uint32_t odd_values;
};
struct SplitWorkspace {
  uint8_t* parts;  // [tile][kSplitTile]
  TileExps* exps;  // [tile]
  int* own;        // [tile][key]: its exponents, the key's below, the value's above
};
constexpr size_t kSplitBytes = kSplitTile + sizeof(TileExps) + kSplitKeys * sizeof(int);  // of a tile

__device__ __forceinline__ float ldexp_f32(float x, int e) { return __builtin_amdgcn_ldexpf(x, e); }

// e with top 2^e in [2^14, 2^15).
__device__ __forceinline__ int unit_exponent(float top, int of_zero) {
  return top > 0.f ? 15 - __builtin_amdgcn_frexp_expf(top) : of_zero;
}
constexpr int kNoValue = 200;     // exponent of values of zero: they scale no others down
constexpr int kOddKey = -0x8000;  // that of a key whose elements are not all finite

// Eight floats times 2^e (2^e[j]) as hi and lo parts.
__device__ __forceinline__ void split_f16(const float* x, const int* e, f16x8_t* hi, f16x8_t* lo) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = ldexp_f32(x[j], e[j]);
    (*hi)[j] = (_Float16)y;
    (*lo)[j] = (_Float16)(y - (float)(*hi)[j]);
  }
}
__device__ __forceinline__ void split_f16(const float* x, int e, f16x8_t* hi, f16x8_t* lo) {
  const int all[8] = {e, e, e, e, e, e, e, e};
  split_f16(x, all, hi, lo);
}

// Tile x of the packed prompts' keys (32 of one prompt; the tiles of prompt b
// start at cu[b] / 32 + b): hi and lo parts of keys and values in the order in
// which the lanes of prompt_attend_f32_kernel take them as operands, and the
// exponents.  Elements that are not finite are zero in the parts, as they would
// reach the rows that do not see them (0 times a NaN is one): their tiles are mixed
// and say where they are.  Reads each element once, writes as many bytes: HBM bound.
__global__ __launch_bounds__(256) void prompt_split_kernel(PromptArgs a, SplitWorkspace ws) {
  __shared__ int part[4][4];
  __shared__ int own_v[kSplitKeys], odd[kSplitKeys];
  __shared__ float vals[kSplitKeys][kHeadDim + 4];
  const int hk = blockIdx.x % a.H_kv, tile = blockIdx.x / a.H_kv;
  const Block blk = find_block(a, tile, 1, kSplitKeys);
  if (blk.len == 0) return;
  const int start = blk.start, len = blk.len, key0 = blk.row0;
  const int tid = threadIdx.x, row = tid / 8, c = tid % 8 * 16;
  float k[16], v[16];
  const bool in = key0 + row < len;
  const size_t tok = (size_t)(start + min(key0 + row, len - 1));
  const float* kp = (const float*)a.k + tok * a.ld_k + (size_t)hk * kHeadDim + c;
  const float* vp = (const float*)a.v + tok * a.ld_v + (size_t)hk * kHeadDim + c;
  float kt = 0.f, vt = 0.f;
  bool odd_k = false, odd_v = false;
#pragma unroll
  for (int j = 0; j < 16; j += 4) {
    const float4 x = *reinterpret_cast<const float4*>(kp + j), y = *reinterpret_cast<const float4*>(vp + j);
    k[j] = x.x, k[j + 1] = x.y, k[j + 2] = x.z, k[j + 3] = x.w;
    v[j] = y.x, v[j + 1] = y.y, v[j + 2] = y.z, v[j + 3] = y.w;
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    if (!in) k[j] = v[j] = 0.f;
    odd_k |= !finite(k[j]);
    odd_v |= !finite(v[j]);
    if (!finite(k[j])) k[j] = 0.f;
    if (!finite(v[j])) v[j] = 0.f;
    kt = fmaxf(kt, fabsf(k[j]));
    vt = fmaxf(vt, fabsf(v[j]));
  }
#pragma unroll
  for (int j = 0; j < 16; j += 4)
    *reinterpret_cast<float4*>(&vals[row][c + j]) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
#pragma unroll
  for (int m = 1; m < 8; m <<= 1) {  // the row's largest
    kt = fmaxf(kt, __shfl_xor(kt, m));
    vt = fmaxf(vt, __shfl_xor(vt, m));
    odd_k |= __shfl_xor((int)odd_k, m);
    odd_v |= __shfl_xor((int)odd_v, m);
  }
  int ek = unit_exponent(kt, 0), ev = unit_exponent(vt, kNoValue);
  // least and largest exponents: of keys that are not zero, of values
  constexpr int kFar = 1 << 20;
  int lim[4] = {kt > 0.f ? ek : kFar, kt > 0.f ? -ek : kFar, in ? ev : kFar, odd_k || odd_v ? -kFar : in ? -ev : kFar};
#pragma unroll
  for (int m = 8; m < kWave; m <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) lim[i] = min(lim[i], __shfl_xor(lim[i], m));
  if (tid % kWave == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i][tid / kWave] = lim[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) lim[i] = min(min(part[i][0], part[i][1]), min(part[i][2], part[i][3]));
  const bool keys = lim[0] != kFar;
  const bool mixed = (keys && -lim[1] - lim[0] > kSpread) || -lim[3] - lim[2] > kSpread;
  const size_t id = (size_t)tile * a.H_kv + hk;
  if (!mixed) ek = keys ? lim[0] : 0, ev = lim[2];
  if (tid % 8 == 0) {
    own_v[row] = ev;
    odd[row] = odd_v;
    ws.own[id * kSplitKeys + row] = ((odd_k ? kOddKey : ek) & 0xffff) | (int)((uint32_t)ev << 16);
  }
  uint8_t* out = ws.parts + id * kSplitTile;
  constexpr int kPart = kSplitTile / 4;
#pragma unroll
  for (int u = 0; u < 2; ++u) {  // dims 16 x + 8 h of key `row`: step x = c / 16, lane 32 h + row
    f16x8_t hi, lo;
    split_f16(k + 8 * u, ek, &hi, &lo);
    const int to = (c / 16) * 1024 + (32 * u + row) * 16;
    __builtin_memcpy(out + to, &hi, 16);
    __builtin_memcpy(out + kPart + to, &lo, 16);
  }
  __syncthreads();  // own_v, odd
  if (tid < kWave) {
    const uint32_t odd_values = (uint32_t)__ballot(tid < kSplitKeys && odd[tid % kSplitKeys]);
    if (tid == 0) ws.exps[id] = TileExps{keys ? lim[0] : 0, lim[2], mixed, odd_values};
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {  // step u, dim block d: lane 32 h + (dim % 32) holds keys 16 u + 4 h + {0..3, 8..11}
    const int d = tid / 64, lane = tid % 64, h = lane / 32;
    float y[8];
    int e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = 16 * u + 4 * h + j % 4 + 8 * (j / 4);
      y[j] = vals[key][32 * d + lane % 32];
      e[j] = own_v[key];
    }
    f16x8_t hi, lo;
    split_f16(y, e, &hi, &lo);
    const int to = (4 * u + d) * 1024 + lane * 16;
    __builtin_memcpy(out + 2 * kPart + to, &hi, 16);
    __builtin_memcpy(out + 3 * kPart + to, &lo, 16);
  }
}

// As prompt_attend_kernel, on tiles of 32 keys in parts; with KS = 2 a step
// stages two tiles and each half of the waves takes one.
//
// Weights are split into fp16 parts too, whose least step is 2^-24: they are
// scaled by what a key adds to the sums, its weight times its largest value, and
// not by the weight alone.  A row behind a sink (a key that takes the weight, its
// value near zero) or behind unattended keys of huge values keeps its 22 bits:
// with c the running maximum of log2(weight) less the values' exponent, a
// weight is held as p 2^(C - e), at most 2^15, where C = 15 - kRoom - (c - m); C is
// a whole number, so that this scaling is exact.  What the parts leave of a weight
// is then 2^-35 of the largest of the row's p 2^-e, and what that takes from the
// sums 2^-30 of its largest p |v| (a tile's tokens are up to 2^kSpread apart).
constexpr float kRoom = 4.f;      // powers of two that c may be passed by before the sums are moved
constexpr int kNothing = 1000;    // C of a row without a key
template <int KS>
__global__ __launch_bounds__(256, 3 - KS) void prompt_attend_f32_kernel(PromptArgs a, SplitWorkspace ws) {
  __shared__ alignas(1024) uint8_t lds_a[KS * kSplitTile], lds_b[KS * kSplitTile];
  constexpr int kPart = kSplitTile / 4, kBlockRows = kRows / KS;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int hk = blockIdx.x % a.H_kv, G = a.H_q / a.H_kv;
  const Block blk = find_block(a, a.tiles - 1 - (int)(blockIdx.x / a.H_kv), G, kBlockRows);
  if (blk.len == 0) return;
  const int n_rows = (int)min((long long)blk.len * G - blk.row0, (long long)kBlockRows);
  const int n = lane % 32, h = lane / 32;
  // this wave's 32 rows and which of a step's KS tiles it takes
  const int rw = KS == 1 ? wave * 32 : wave % 2 * 32, b0 = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave / 2);
  const int row = min(rw + n, n_rows - 1) + blk.row0;
  const int pos = row / G;
  const float* qp = (const float*)a.q + (size_t)(blk.start + pos) * a.ld_q + (size_t)(hk * G + row % G) * kHeadDim;
  f16x8_t qh[8], ql[8];
  int eq;
  {
    float x[64], top = 0.f;  // dims 16 s + 8 h .. + 7
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      const float4 v = *reinterpret_cast<const float4*>(qp + 16 * (s / 2) + 8 * h + 4 * (s % 2));
      x[4 * s] = v.x, x[4 * s + 1] = v.y, x[4 * s + 2] = v.z, x[4 * s + 3] = v.w;
    }
#pragma unroll
    for (int j = 0; j < 64; ++j) top = fmaxf(top, fabsf(x[j]));
    eq = unit_exponent(fmaxf(top, swap32(top)), 0);
#pragma unroll
    for (int s = 0; s < 8; ++s) split_f16(x + 8 * s, eq, &qh[s], &ql[s]);
  }
  const int pos_lo = (blk.row0 + min(rw, n_rows - 1)) / G;
  const int pos_hi = (blk.row0 + min(rw + 31, n_rows - 1)) / G;
  const int n_tiles = (blk.row0 + n_rows - 1) / G / kSplitKeys + 1;
  const size_t tile0 = ((size_t)(blk.start / kSplitKeys + blk.b)) * a.H_kv + hk;
  auto stage = [&](int step, uint8_t* to) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const int t = min(step * KS + j, n_tiles - 1);
      const uint8_t* p = ws.parts + (tile0 + (size_t)t * a.H_kv) * kSplitTile + wave * 8192 + lane * 16;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        __builtin_amdgcn_global_load_lds((global_void*)(p + u * 1024),
                                         (lds_void*)(to + j * kSplitTile + wave * 8192 + u * 1024), 16, 0, 0);
    }
  };
  const int n_steps = (n_tiles + KS - 1) / KS;

  f32x16_t o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  // m: the running maximum in powers of two, that of the weights' sum l; o holds
  // sums of p times the values times 2^C
  float m = -INFINITY, c = -INFINITY, l = 0.f;
  int C = kNothing;
  auto tile = [&](int step, const uint8_t* kt, uint8_t* next, auto mixed) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's part of the step's tiles
    __syncthreads();
    if (step + 1 < n_steps) stage(step + 1, next);
    const int t = step * KS + b0;
    if (t * kSplitKeys > pos_hi) return;
    kt += b0 * kSplitTile;
    const TileExps ex = ws.exps[tile0 + (size_t)t * a.H_kv];
    kt += lane * 16;
    f32x16_t s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      f16x8_t kh, kl;
      __builtin_memcpy(&kh, kt + x * 1024, 16);
      __builtin_memcpy(&kl, kt + kPart + x * 1024, 16);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kl, qh[x], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh, ql[x], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh, qh[x], s, 0, 0, 0);
    }
    int own[16];
    if constexpr (mixed) {
      const int* p = ws.own + (tile0 + (size_t)t * a.H_kv) * kSplitKeys + 4 * h;
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(own + 4 * i, p + 8 * i, 16);
    }
    auto own_k = [&](int i) { return (int)(short)own[i]; };
    auto own_v = [&](int i) { return own[i] >> 16; };
    // (in range, so that neither 0 times it nor -inf times it is a NaN)
    auto factor = [&](int e) { return fminf(fmaxf(ldexp_f32(kScale * kLog2e, -(eq + e)), 0x1p-120f), 0x1p120f); };
    float f = 1.f;
    if constexpr (mixed) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = own_k(i) == kOddKey ? NAN : s[i] * factor(own_k(i));
    } else {
      f = factor(ex.k);
    }
    if (t * kSplitKeys + kSplitKeys - 1 > pos_lo) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (t * kSplitKeys + 8 * (i / 4) + 4 * h + i % 4 > pos) s[i] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = fmaxf(top, swap32(top)) * f;
    float adds = top - (float)ex.v;
    if constexpr (mixed) {
      adds = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) adds = fmaxf(adds, s[i] - (float)own_v(i));
      adds = fmaxf(adds, swap32(adds));
    }
    if (__any(top > m + kSlack || adds > c + kRoom)) {
      const float m1 = fmaxf(m, top);
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= keep;
      c = fmaxf(c, adds);
      const float apart = fminf(fmaxf(c - m, -400.f), 400.f);  // (a row of NaN or infinities: any)
      const int C1 = m == -INFINITY ? kNothing : (int)floorf(15.f - kRoom - apart);
      const float turn = ldexp_f32(keep, C1 - C);
      C = C1;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= turn;
    }
    const float shift = m == -INFINITY ? 0.f : -m;
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], f, shift));
      l += p[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = ldexp_f32(p[i], C - (mixed ? own_v(i) : ex.v));  // (2^(C - e) may not be a float)
    f16x8_t ph[2], pl[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      ph[i / 8][i % 8] = (_Float16)p[i];
      pl[i / 8][i % 8] = (_Float16)(p[i] - (float)ph[i / 8][i % 8]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f16x8_t vh, vl;
        __builtin_memcpy(&vh, kt + 2 * kPart + (4 * x + d) * 1024, 16);
        __builtin_memcpy(&vl, kt + 3 * kPart + (4 * x + d) * 1024, 16);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vl, ph[x], o[d], 0, 0, 0);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh, pl[x], o[d], 0, 0, 0);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh, ph[x], o[d], 0, 0, 0);
      }
    if constexpr (mixed)
      for (uint32_t odd = ex.odd_values; odd; odd &= odd - 1) {
        const int u = t * kSplitKeys + __builtin_ctz(odd);
        if (__builtin_expect(u <= pos, 0)) add_odd((const float*)a.v + (size_t)(blk.start + u) * a.ld_v + hk * kHeadDim + 4 * h, o);
      }
  };
  // Mixed tiles have a loop of their own (their weights in the same loop took 2 to
  // 15% from all, or spilled), entered by two steps whose tiles are among them; said
  // to be rare, so that it stands apart from the other one (5% of its time)
  uint64_t mixed_tiles = 0;  // of the 64 that this step's are among
  auto mixed_next = [&](int step) {
    const int t = step * KS;
    if (t % kWave == 0)
      mixed_tiles = __ballot(ws.exps[tile0 + (size_t)min(t + lane, n_tiles - 1) * a.H_kv].mixed != 0);
    return (mixed_tiles >> (t % kWave) & ((1u << 2 * KS) - 1)) != 0;
  };
  auto two_steps = [&](int step, auto mixed) __attribute__((always_inline)) {
    tile(step, lds_a, lds_b, mixed);
    if (step + 1 < n_steps) tile(step + 1, lds_b, lds_a, mixed);
  };
  bool mix = mixed_next(0);
  stage(0, lds_a);
  for (int step = 0; step < n_steps;) {
    for (; step < n_steps && __builtin_expect(!mix, 1); step += 2, mix = mixed_next(step)) two_steps(step, std::false_type());
    for (; step < n_steps && __builtin_expect(mix, 0); step += 2, mix = mixed_next(step)) two_steps(step, std::true_type());
  }
  l += swap32(l);
  if constexpr (KS == 2) {  // the second waves' sums join the first ones', through the tiles' memory
    __syncthreads();
    float* x = (float*)(rw ? lds_b : lds_a);  // [64 sums][lane]
    __shared__ float ml[2][2][kWave];
    __shared__ int cs[2][kWave];
    if (b0 == 1) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(16 * d + i) * kWave + lane] = o[d][i];
      ml[rw / 32][0][lane] = m;
      ml[rw / 32][1][lane] = l;
      cs[rw / 32][lane] = C;
    }
    __syncthreads();
    if (b0 == 1) return;
    const float m2 = ml[rw / 32][0][lane], l2 = ml[rw / 32][1][lane], m1 = fmaxf(m, m2);
    const int C2 = cs[rw / 32][lane], C1 = min(C, C2);  // (a row's first key is in the first waves' part)
    float e1 = __builtin_amdgcn_exp2f(m - m1), e2 = __builtin_amdgcn_exp2f(m2 - m1);
    l = l * e1 + l2 * e2;
    e1 = ldexp_f32(e1, C1 - C);
    e2 = ldexp_f32(e2, C1 - C2);
    C = C1;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * e1 + x[(16 * d + i) * kWave + lane] * e2;
  }
  const float inv = 1.f / l;
  if (rw + n < n_rows) {
    float* out = (float*)a.out + ((size_t)(blk.start + pos) * a.H_q + hk * G + row % G) * kHeadDim;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = ldexp_f32(o[d][i + j] * inv, -C);
        *reinterpret_cast<float4*>(out + 32 * d + 2 * i + 4 * h) = make_float4(y[0], y[1], y[2], y[3]);
      }
  }
}

// Token rows of H heads at `p`, ld elements apart: what the 16-byte accesses need.
bool rows_ok(const void* p, size_t ld, int H, int dtype) {
  return p && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld >= (size_t)H * kHeadDim &&
         ld * (dtype == SAKI_F32 ? 4 : 2) % 16 == 0;
}

// Whether blocks of half the rows, whose waves take a tile's keys in two parts,
// are the better ones: a block's time halves, but not the work before and after
// its tiles, so that it needs CUs without a block of their own and keys to part.
// us, whole / halved, prompts x tokens of H_q / H_kv heads:
//                        blocks    bf16           float32
//   4 x 64, 32 / 8           96     8.0 / 7.7     15.4 / 13.7
//   6 x 128, 32 / 8         240     8.7 / 9.3     20.9 / 25.0
//   2 x 400, 32 / 8         216    13.0 / 13.0    33.2 / 28.7
//   4 x 400, 32 / 8         432    18.2 / 21.2    42.6 / 51.9
//   3000, 8 / 8             192    58.2 / 42.4   165.6 / 95.3
//   1200, 28 / 4            264    28.8 / 23.2    69.7 / 62.1
//   4 x 300, 28 / 4         276    12.8 / 13.2    29.9 / 35.6
//   3 x 1000, 12 / 1        284    25.9 / 22.5    62.0 / 65.1
//   6000, 8 / 8             376   122.2 / 98.0   336.8 / 304.5
//   6 x 1024, 8 / 8         432    30.0 / 32.2    86.5 / 92.1
bool halves_better(long long blocks, int T, int B) {
  const int keys = T / B;  // of a prompt, on average
  return blocks <= (keys >= 1000 ? 384 : keys >= 256 ? 224 : 128);
}

constexpr size_t kMaxLd = 1 << 22;  // a tile's byte offsets fit 32 bits

// Tiles of float32 parts that all prompts have, at most.
long long split_tiles(int T, int B) { return (long long)T / kSplitKeys + B; }

}  // namespace

extern "C" {

size_t saki_attend_prompt_workspace_bytes(int dtype, int T, int B, int H_kv) {
  if (T < 0 || B < 0 || H_kv <= 0 || (dtype != SAKI_F32 && dtype != SAKI_BF16)) return 0;
  if (dtype == SAKI_BF16 || T == 0 || B == 0) return 256;
  return (size_t)split_tiles(T, B) * H_kv * kSplitBytes;
}

int saki_attend_prompt(const void* q, const void* k, const void* v, int dtype, int T, int B, int H_q, int H_kv,
                       int d, size_t ld_q, size_t ld_k, size_t ld_v, const int* cu, void* out, void* ws,
                       size_t ws_bytes, void* stream) {
  if (T < 0 || B < 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || d <= 0) return SAKI_ERR_ARG;
  if (d != kHeadDim || (dtype != SAKI_F32 && dtype != SAKI_BF16)) return SAKI_ERR_UNSUPPORTED;
  // row numbers of a KV head fit an int, a launch's threads 32 bits
  const long long rows = (long long)T * (H_q / H_kv);
  long long tiles = rows / kRows + B;  // of whole blocks
  if (rows > INT_MAX / 2 || B > INT_MAX / 2 || 2 * tiles * H_kv > (1 << 23) || split_tiles(T, B) * H_kv > (1 << 23))
    return SAKI_ERR_UNSUPPORTED;
  if (T == 0 || B == 0) return SAKI_OK;
  if (!cu || !out || reinterpret_cast<uintptr_t>(out) % 16 || !rows_ok(q, ld_q, H_q, dtype) ||
      !rows_ok(k, ld_k, H_kv, dtype) || !rows_ok(v, ld_v, H_kv, dtype))
    return SAKI_ERR_ARG;
  if (ld_q > kMaxLd || ld_k > kMaxLd || ld_v > kMaxLd) return SAKI_ERR_UNSUPPORTED;
  const bool halves = halves_better(tiles * H_kv, T, B);
  if (halves) tiles = rows / (kRows / 2) + B;
  const PromptArgs a{q, k, v, ld_q, ld_k, ld_v, cu, B, H_q, H_kv, T, out, (int)tiles};
  const dim3 grid((unsigned)(tiles * H_kv));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == SAKI_BF16) {
    if (halves)
      hipLaunchKernelGGL((prompt_attend_kernel<2>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((prompt_attend_kernel<1>), grid, dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? SAKI_OK : SAKI_ERR_HIP;
  }
  if (!ws || ws_bytes < saki_attend_prompt_workspace_bytes(dtype, T, B, H_kv) || reinterpret_cast<uintptr_t>(ws) % 16)
    return SAKI_ERR_WORKSPACE;
  const long long n = split_tiles(T, B) * H_kv;
  SplitWorkspace w;  // the exponents stand behind the parts
  w.parts = (uint8_t*)ws;
  w.exps = (TileExps*)(w.parts + (size_t)n * kSplitTile);
  w.own = (int*)(w.exps + n);
  hipLaunchKernelGGL(prompt_split_kernel, dim3((unsigned)n), dim3(256), 0, s, a, w);
  if (hipGetLastError() != hipSuccess) return SAKI_ERR_HIP;
  if (halves)
    hipLaunchKernelGGL((prompt_attend_f32_kernel<2>), grid, dim3(256), 0, s, a, w);
  else
    hipLaunchKernelGGL((prompt_attend_f32_kernel<1>), grid, dim3(256), 0, s, a, w);
  return hipGetLastError() == hipSuccess ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"
