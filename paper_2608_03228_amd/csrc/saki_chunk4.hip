// Causal attention of prompts that continue a 4-bit cache, for gfx950 (CDNA4, wave64):
//
//   cache4_prompt_kernel  packed chunks of new tokens over all that the cache holds
//   cache4_gather_kernel  joins the parts of rows whose keys several work-groups shared

#include "saki_cache4.h"
#include "saki_rows.h"

namespace {

using saki_dev::Block;

typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kScale = 0.08838834764831845f;  // 1 / sqrt(d)
constexpr int kRows = 128;                      // query rows of a work-group (32 a wave), or half of them
// A row's sums are scaled down only once a score passes the maximum they go by
// by this many powers of two.
constexpr float kSlack = 8.f;
constexpr size_t chunk_part(int rows) { return (size_t)rows * (kHeadDim + 2); }  // floats: sums, maxima, weights

struct Chunk4Args {
  const void* q;
  size_t ld_q;
  const uint8_t *k, *v, *scales;
  int n_blocks;
  const int* tables;
  int max_blocks;
  const int *lens, *cu;
  int B, H_q, H_kv, T;
  void* out;
  int splits;  // work-groups that share a row block's keys
};

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ float swap32(float v) { return xor_f32(v, 32); }

// out_t = sum_u p_u v_u over the cached keys up to token t's position.  A
// work-group takes 128 (token, query head) rows of one KV head, 32 a wave, and
// goes through the keys in the cache's blocks of 64: each thread holds 16 bytes of
// the next block's keys and values, converts them to bf16 with their scales
// (exactly) and puts them into LDS, two blocks deep, while the block before is
// multiplied.  Two groups a CU fill each other's pauses.  S^T = K Q^T leaves a lane
// with scores of one row, so the softmax is in registers but for one exchange, and
// its weights are at once the operand of O^T = V^T P^T, whose other operand the
// transposing LDS reads form.  bf16: weights rounded to bf16, which takes a row's error
// from 0.0016 of it (its output's rounding) to 0.0018-0.0019; a second term would be as
// many products again as the values take now.  float32: queries and weights in three
// bf16 terms, 32 keys at a time for the registers' sake.
//
// Bound by power and the MFMA, with the softmax beside it: 2,000 tokens of 32 / 8
// heads over 23,000 and 32,800 keys in 950-1,060 us, 0.88-0.98 PFLOP/s depending on
// the card (a large bf16 matrix product reaches 1.17-1.27), the MFMA 41% busy, and a
// whole prompt of 8,192 in 605, 0.91; float32, three products each, 0.36 PFLOP/s (the
// prompt 0.39).  256 rows a work-group, which halves
// the conversions, took as long.
//
// KS = 2: 64 rows, and two waves share a row's keys, 32 of each block; their sums
// meet at the end (see chunk_plan).
template <bool F32, bool SPLIT, int KS>
__global__ __launch_bounds__(256, 2) void cache4_prompt_kernel(Chunk4Args a, float* __restrict__ ws) {
  using T = std::conditional_t<F32, float, __bf16>;
  constexpr int kQT = F32 ? 3 : 1;
  constexpr int NB = F32 || KS == 2 ? 1 : 2;  // 32 keys each, between two looks at the maximum
  constexpr int kBlockRows = kRows / KS;
  constexpr int kTileBytes = kTile * kHeadDim * 2;
  // two arrays, and the loop below unrolled over them: a read of one is then known
  // not to meet the writes to the other
  __shared__ alignas(1024) uint8_t lds_a[2 * kTileBytes], lds_b[2 * kTileBytes];  // keys, values
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int hk = blockIdx.x % a.H_kv, G = a.H_q / a.H_kv;
  const int part = blockIdx.x / a.H_kv, sp = SPLIT ? part % a.splits : 0, x = SPLIT ? part / a.splits : part;
  const Block blk = saki_dev::find_block(a.cu, a.B, a.T, x, G, kBlockRows);
  if (blk.len == 0) return;
  const int n_rows = (int)min((long long)blk.len * G - blk.row0, (long long)kBlockRows);
  const int n = lane % 32, h = lane / 32, rw = wave % (4 / KS) * 32;

  // this lane's row, its token, head and position; the least and largest position
  // of the group's rows and of the wave's
  const int row = min(rw + n, n_rows - 1) + blk.row0, tok = row / G;
  // the first row's position: a request's last token stands at lens - 1, also where its offsets end past the T
  // tokens of the call.  (A length near the lowest int stands for none, as others below zero do.)
  const int before = (int)max((long long)a.lens[blk.b] - a.cu[blk.b + 1] + blk.start, -(1LL << 30));
  const int pos = before + tok;
  const int pos_min = before + blk.row0 / G, pos_max = before + (blk.row0 + n_rows - 1) / G;
  const int pos_lo = before + (blk.row0 + min(rw, n_rows - 1)) / G;
  const int pos_hi = before + (blk.row0 + min(rw + 31, n_rows - 1)) / G;
  const int nt = tiles_of(pos_max + 1, a.max_blocks);
  const int piece = SPLIT ? (nt + a.splits - 1) / a.splits : nt;
  const int t0 = sp * piece, t1 = min(nt, t0 + piece);

  bf16x8_t q[8][kQT];  // dims 16 x + 8 h ..
  {
    const T* p = (const T*)a.q + (size_t)(blk.start + tok) * a.ld_q + (size_t)(hk * G + row % G) * kHeadDim + 8 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if constexpr (F32) {
        float y[8];
        load_elems<float, 8>(p + 16 * s, y);
        split_bf16<kQT>(y, q[s]);
      } else {
        const uint4 y = *reinterpret_cast<const uint4*>(p + 16 * s);
        __builtin_memcpy(&q[s][0], &y, 16);
      }
    }
  }

  const const_int* table = (const const_int*)(uintptr_t)(a.tables + (size_t)blk.b * a.max_blocks);
  auto block_of = [&](int t) __attribute__((always_inline)) {
    const int at = t < t1 ? table[t] : -1;
    return at < a.n_blocks ? at : -1;  // (below 0: none)
  };
  // a thread's share of a block: group tid % 4 of key tid / 4; dims 8 (tid % 16) .. of tokens 4 (tid / 16) ..
  uint4 kx, vx, vs;
  uint32_t ks;
  auto fetch = [&](int at) __attribute__((always_inline)) {
    if (at < 0) return;
    const size_t i = (size_t)at * a.H_kv + hk;
    kx = *reinterpret_cast<const uint4*>(a.k + i * kCodes4 + tid * 16);
    vx = *reinterpret_cast<const uint4*>(a.v + i * kCodes4 + tid * 16);
    ks = a.scales[i * kScales4 + tid];
    vs = *reinterpret_cast<const uint4*>(a.scales + i * kScales4 + kTile * kGroups4 + tid / 16 * 16);
  };
  // bf16 rows of 16 pieces: piece c of key row r at place c ^ (r % 16), of value row r at c ^ (r % 4 * 4)
  auto put = [&](int t, uint8_t* to) __attribute__((always_inline)) {
    const uint32_t kc[4] = {kx.x, kx.y, kx.z, kx.w}, vc[4] = {vx.x, vx.y, vx.z, vx.w}, ve[4] = {vs.x, vs.y, vs.z, vs.w};
    const int r = tid / 4, v0 = tid / 16 * 4, turn = (tid % 16 / 4 * 8 + 9) % 32;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint32_t w[4];
      decode8(kc[s], scale_of(ks), w);
      *reinterpret_cast<uint4*>(to + r * 256 + (((tid % 4 * 4 + s) ^ (r % 16)) * 16)) =
          make_uint4(w[0], w[1], w[2], w[3]);
    }
    float f[4];  // (the conversion reads the exponent alone)
#pragma unroll
    for (int c = 0; c < 4; ++c) f[c] = __uint_as_float(__builtin_amdgcn_alignbit(ve[c], ve[c], turn));
    if (t * kTile + kTile - 1 > pos_min) {
      // a weight of zero has to make them zero: tokens that no row sees, and NaN where a row may not see it (below)
      int u = t * kTile + v0;
      asm volatile("" : "+v"(u));  // (what follows stays in the branch)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (u + c > pos_max || (u + c > pos_min && (__float_as_uint(f[c]) & 0x7f800000u) == 0x7f800000u)) f[c] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t w[4];
      decode8(vc[c], f[c], w);
      *reinterpret_cast<uint4*>(to + kTileBytes + (v0 + c) * 256 + (((tid % 16) ^ (c * 4)) * 16)) =
          make_uint4(w[0], w[1], w[2], w[3]);
    }
  };

  f32x16_t o[4];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  const int k_lane = n * 256 + ((h ^ (lane % 16)) * 16);
  const int ls = lane % 16, lg = lane / 16;
  const int v_lane = (4 * (lg / 2) + ls / 4) * 256 + 32 * (lg % 2) + 8 * (ls % 4);

  auto tile = [&](int t, const uint8_t* kt) __attribute__((always_inline)) {
    if (rw >= n_rows || t * kTile > pos_hi) return;
    const uint8_t* vt = kt + kTileBytes;
#pragma unroll
    for (int half = 0; half < 2 / KS; half += NB) {
      const int b0 = KS == 2 ? wave / 2 : half;
      f32x16_t s[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          bf16x8_t kf;
          __builtin_memcpy(&kf, kt + (b + b0) * 32 * 256 + (k_lane ^ (y * 32)), 16);
#pragma unroll
          for (int z = kQT - 1; z >= 0; --z) s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[y][z], s[b], 0, 0, 0);
        }
      }
      if (t * kTile + kTile - 1 > pos_lo) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (t * kTile + 32 * (b + b0) + 8 * (i / 4) + 4 * h + i % 4 > pos) s[b][i] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 16 * NB; ++i) top = fmaxf(top, s[i / 16][i % 16]);
      top = fmaxf(top, swap32(top));
      if (__any(top > m + kSlack / (kScale * kLog2e))) {
        const float m1 = fmaxf(m, top);
        float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m1) * (kScale * kLog2e));
        asm volatile("" : "+v"(keep));  // (the products below stay in the branch)
        m = m1;
        l *= keep;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= keep;
      }
      const float shift = m == -INFINITY ? 0.f : -m * (kScale * kLog2e);  // (a row that sees none of the keys yet)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float sum = 0.f;  // (a sum of sums: a row's N / 2 weights one by one would lose 2^-24 sqrt(N) of it)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], kScale * kLog2e, shift));
          sum += s[b][i];
        }
        l += sum;
      }
#pragma unroll
      for (int y = 0; y < 2 * NB; ++y) {  // 16 keys each
        float p[8];
        bf16x8_t pt[kQT];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = s[y / 2][y % 2 * 8 + i];
        split_bf16<kQT>(p, pt);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
          const uint8_t* at = vt + (y + 2 * b0) * 16 * 256 + (v_lane ^ ((d ^ (ls / 4)) * 64));
          const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds_void*)at);
          const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds_void*)(at + 8 * 256));
          bf16x8_t vf;
          __builtin_memcpy(&vf, &lo, 8);
          __builtin_memcpy((char*)&vf + 8, &hi, 8);
#pragma unroll
          for (int z = kQT - 1; z >= 0; --z) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pt[z], o[d], 0, 0, 0);
        }
      }
    }
  };

  int at0 = block_of(t0), at1 = block_of(t0 + 1), at2 = block_of(t0 + 2);
  fetch(at0);
  if (at0 >= 0) put(t0, lds_a);
  // the queries are there: waited for in the loop, they would have it wait for the next block too (with tables
  // read by vector loads, 1.05 us for 0.88 a block of 64 rows)
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  fetch(at1);
  if constexpr (!F32) {
    // a row with an infinite query is NaN, but products alone may give one infinity for all its scores, which are
    // a row without a key then: one element NaN makes them NaN (the terms of float32 do so by themselves)
    uint32_t odd = 0;  // the top bit of a half: an exponent of ones
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      uint32_t w[4];
      __builtin_memcpy(w, &q[s][0], 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= (w[e] & 0x7f807f80u) + 0x00800080u;
    }
    if (odd & 0x80008000u) q[0][0][0] = (__bf16)NAN;
  }
  auto step = [&](int t, const uint8_t* now, uint8_t* next) __attribute__((always_inline)) {
    __syncthreads();  // block t is in `now`, and `next` is read
    const int at3 = block_of(t + 3);
    if (at1 >= 0) put(t + 1, next);
    fetch(at2);
    if (at0 >= 0) tile(t, now);
    at0 = at1;
    at1 = at2;
    at2 = at3;
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, lds_a, lds_b);
    if (t + 1 < t1) step(t + 1, lds_b, lds_a);
  }

  // NaN for the rows that see a value that is one and that some row of the group
  // does not see, in its group's dims: o[d] holds group d
  for (int t = max(t0, max(pos_min, 0) / kTile); t < t1; ++t) {
    const int at = block_of(t);
    if (at < 0) continue;
    const uint32_t e = *reinterpret_cast<const uint32_t*>(a.scales + ((size_t)at * a.H_kv + hk) * kScales4 +
                                                          (kTile + lane) * kGroups4);
    const int left = pos - t * kTile + 1;  // tokens of the block that this lane's row sees
    const uint64_t sees = left <= 0 ? 0 : left >= 64 ? ~0ull : (1ull << left) - 1;
#pragma unroll
    for (int d = 0; d < 4; ++d)
      if (__ballot((e >> (8 * d) & 255) == 255) & sees) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = NAN;
      }
  }

  l += swap32(l);
  if constexpr (KS == 2) {  // the second waves' sums join the first ones', through the blocks' memory
    __syncthreads();        // all blocks are read
    float* y = (float*)(rw ? lds_b : lds_a);  // [64 sums][lane]
    static_assert(2 * kTileBytes >= 64 * kWave * 4);
    __shared__ float ml[2][2][kWave];
    if (wave >= 2) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[(16 * d + i) * kWave + lane] = o[d][i];
      ml[rw / 32][0][lane] = m;
      ml[rw / 32][1][lane] = l;
    }
    __syncthreads();
    if (wave >= 2) return;
    const float m2 = ml[rw / 32][0][lane], l2 = ml[rw / 32][1][lane], m1 = fmaxf(m, m2);
    const float ref = m1 == -INFINITY ? 0.f : m1;
    const float e1 = __builtin_amdgcn_exp2f((m - ref) * (kScale * kLog2e));
    const float e2 = __builtin_amdgcn_exp2f((m2 - ref) * (kScale * kLog2e));
    m = m1;
    l = l * e1 + l2 * e2;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * e1 + y[(16 * d + i) * kWave + lane] * e2;
  }
  if (rw + n >= n_rows) return;
  if constexpr (SPLIT) {
    float* w = ws + ((size_t)(x * a.H_kv + hk) * a.splits + sp) * chunk_part(kBlockRows);
    if (h == 0) w[kBlockRows * kHeadDim + rw + n] = m, w[kBlockRows * (kHeadDim + 1) + rw + n] = l;
    if (t0 >= t1) return;
    w += (rw + n) * kHeadDim + 4 * h;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(w + 32 * d + 2 * i) = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
  } else {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* to = (T*)a.out + ((size_t)(blk.start + tok) * a.H_q + hk * G + row % G) * kHeadDim + 4 * h;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        if constexpr (F32)
          *reinterpret_cast<float4*>(to + 32 * d + 2 * i) =
              make_float4(o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv);
        else
          *reinterpret_cast<uint2*>(to + 32 * d + 2 * i) =
              make_uint2(pack_bf16(o[d][i] * inv, o[d][i + 1] * inv), pack_bf16(o[d][i + 2] * inv, o[d][i + 3] * inv));
      }
  }
}

// Joins a row's parts.  LANES = 64: a wave a row; its lanes hold the parts' maxima
// and weights, 64 at a time, then half of the wave sums every second part, 4 dims a
// lane, eight parts' loads at once (a part after another, 51 parts of 100 tokens
// over 32,768 keys of one head took 50 us).  LANES = 16, for up to 6 parts: four rows
// a wave, 8 dims a lane (two parts of 28,672 float32 rows: 5.5 us less).
template <bool F32, int KS, int LANES>
__global__ __launch_bounds__(256) void cache4_gather_kernel(Chunk4Args a, const float* __restrict__ ws) {
  using T = std::conditional_t<F32, float, __bf16>;
  constexpr int kBlockRows = kRows / KS, kAtOnce = 4;
  constexpr int kDims = LANES == 64 ? 4 : 8, kSide = LANES * kDims / kHeadDim;  // parts side by side
  constexpr size_t kPart = chunk_part(kBlockRows);
  const int c = threadIdx.x % LANES, side = c / (kHeadDim / kDims), d0 = c % (kHeadDim / kDims) * kDims;
  const int first = threadIdx.x % kWave - c;  // the row's lanes
  const int hk = blockIdx.x % a.H_kv, x = blockIdx.x / a.H_kv, G = a.H_q / a.H_kv;
  const Block blk = saki_dev::find_block(a.cu, a.B, a.T, x, G, kBlockRows);
  const int i = blockIdx.y * (256 / LANES) + threadIdx.x / LANES;
  const bool in = i < (long long)blk.len * G - blk.row0;
  if (blk.len == 0 || !__any(in)) return;
  const float* w = ws + (size_t)(x * a.H_kv + hk) * a.splits * kPart;
  const float *wm = w + kBlockRows * kHeadDim + i, *wl = wm + kBlockRows;
  const int parts = in ? a.splits : 0;
  float M = -INFINITY;
  for (int s = c; s < parts; s += LANES) M = fmaxf(M, wm[s * kPart]);
#pragma unroll
  for (int y = 1; y < LANES; y <<= 1) M = fmaxf(M, xor_f32(M, y));
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f, sum[kDims];
#pragma unroll
  for (int d = 0; d < kDims; ++d) sum[d] = 0.f;
  for (int s0 = 0; s0 < a.splits; s0 += LANES) {
    const int n = min(a.splits - s0, LANES);
    // a part's factor; below 0: no key of it is seen, and its sums may never have been written.  A factor of zero
    // is another matter (keys that score far below the others): its sums may be NaN, and the row is then, too
    float e = -1.f;
    if (s0 + c < parts) {
      const float l = wl[(s0 + c) * kPart];
      if (l != 0.f) e = __builtin_amdgcn_exp2f((wm[(s0 + c) * kPart] - ref) * (kScale * kLog2e)), L += l * e;
    }
    for (int s = 0; s < n; s += kSide * kAtOnce) {
      float z[kAtOnce][kDims], f[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int t = s + kSide * u + side;
        f[u] = __shfl(e, first + t % LANES);
#pragma unroll
        for (int d = 0; d < kDims; ++d) z[u][d] = 0.f;
        if (t < n && !(f[u] < 0.f)) load_elems<float, kDims>(w + (s0 + t) * kPart + i * kHeadDim + d0, z[u]);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
        for (int d = 0; d < kDims; ++d) sum[d] += z[u][d] * f[u];
    }
  }
#pragma unroll
  for (int y = 1; y < LANES; y <<= 1) L += xor_f32(L, y);
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int d = 0; d < kDims; ++d) {
    if constexpr (kSide == 2) sum[d] += xor_f32(sum[d], 32);
    sum[d] *= inv;
  }
  const int row = blk.row0 + i;
  if (in && side == 0)
    store_elems<T, kDims>((T*)a.out + ((size_t)(blk.start + row / G) * a.H_q + hk * G + row % G) * kHeadDim + d0, sum);
}

// How a call is divided.
struct ChunkPlan {
  bool halves;       // 64 rows a work-group
  long long groups;  // row blocks of the packed tokens (at most) times KV heads
  int splits;        // work-groups that share a block's keys
  size_t ws_bytes() const {
    return splits > 1 ? (size_t)groups * splits * chunk_part(halves ? kRows / 2 : kRows) * sizeof(float) : 256;
  }
};

// Row blocks that hold rows, more or less: a request has one at least, its last one half full.
long long blocks_of(long long rows, int block_rows, int B) {
  const long long n = rows / block_rows + (B + 1) / 2;
  return n > B ? n : B;
}

// Which blocks and how many shares take the least time, by what one cache block
// takes a work-group: us, alone on a CU and beside another (256 and 512 groups
// over 16,384 tokens and more),
//              bf16           float32
//   128 rows   1.28 / 2.04    2.88 / 4.85
//    64 rows   0.88 / 1.31    1.65 / 2.65
// and the join: 4 us, and a part written and read.  The tables' width stands for
// the lengths, which are on the device.
ChunkPlan chunk_plan(int dtype, int T, int B, int G, int H_kv, int max_blocks) {
  static const float kTake[2][2][2] = {{{2.88f, 4.85f}, {1.65f, 2.65f}}, {{1.28f, 2.04f}, {0.88f, 1.31f}}};
  const long long rows = (long long)T * G;
  ChunkPlan best{false, 0, 0};
  float least = 0.f;
  for (int halves = 0; halves < 2; ++halves) {
    const int block_rows = halves ? kRows / 2 : kRows;
    const float* take = kTake[dtype == SAKI_BF16][halves];
    const long long n = blocks_of(rows, block_rows, B) * H_kv;
    const long long shares[4] = {1, 256 / n, 512 / n, 1024 / n};
    for (int i = 0; i < 4; ++i) {
      const long long most = max_blocks < 4 ? 1 : max_blocks / 2;  // two blocks each at least
      const long long s = shares[i] < most ? shares[i] : most;
      if (i && s <= 1) continue;
      const long long all = n * s, rest = all % 512;
      const float each = (float)((max_blocks + s - 1) / s);
      float us = each * ((float)(all / 512) * take[1] + (rest == 0 ? 0.f : take[rest > 256]));
      if (s > 1) us += 4.f + (float)all * (float)block_rows * 2.1e-4f;
      if (best.groups == 0 || us < least) {
        least = us;
        best = ChunkPlan{halves == 1, (rows / block_rows + B) * H_kv, (int)s};
      }
    }
  }
  return best;
}

template <bool F32, int KS>
int launch_chunk(const ChunkPlan& p, const Chunk4Args& a, void* ws, hipStream_t s) {
  const dim3 grid((unsigned)(p.groups * p.splits));
  if (p.splits == 1) {
    hipLaunchKernelGGL((cache4_prompt_kernel<F32, false, KS>), grid, dim3(256), 0, s, a, nullptr);
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  hipLaunchKernelGGL((cache4_prompt_kernel<F32, true, KS>), grid, dim3(256), 0, s, a, (float*)ws);
  if (!launched()) return SAKI_ERR_HIP;
  if (p.splits <= 6)
    hipLaunchKernelGGL((cache4_gather_kernel<F32, KS, 16>), dim3((unsigned)p.groups, kRows / KS / 16), dim3(256), 0, s,
                       a, (const float*)ws);
  else
    hipLaunchKernelGGL((cache4_gather_kernel<F32, KS, 64>), dim3((unsigned)p.groups, kRows / KS / 4), dim3(256), 0, s,
                       a, (const float*)ws);
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // namespace

extern "C" {

size_t saki_cache4_prompt_workspace_bytes(int dtype, int T, int B, int H_q, int H_kv, int max_blocks) {
  if (T < 0 || B < 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || max_blocks <= 0 || !type_ok(dtype))
    return 0;
  if (T == 0 || B == 0) return 256;
  return chunk_plan(dtype, T, B, H_q / H_kv, H_kv, max_blocks).ws_bytes();
}

int saki_cache4_prompt(const void* q, int dtype, int T, int B, int H_q, int H_kv, int d, size_t ld_q,
                       const void* k_cache, const void* v_cache, const void* scales, int n_blocks, const int* tables,
                       int max_blocks, const int* lens, const int* cu, void* out, void* ws, size_t ws_bytes,
                       void* stream) {
  if (T < 0 || B < 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || d <= 0 || max_blocks <= 0) return SAKI_ERR_ARG;
  const int st = check_cache4(k_cache, v_cache, scales, n_blocks, H_kv);
  if (st != SAKI_OK) return st;
  const int G = H_q / H_kv;
  if (d != kHeadDim || !type_ok(dtype) || T > kMaxTokens || B > INT_MAX / 2 || max_blocks > INT_MAX / kTile - 1 ||
      (long long)T * G >= INT_MAX / 2 || 2 * ((long long)T * G / kRows + B) * H_kv > (1 << 23) || H_q > 65535)
    return SAKI_ERR_UNSUPPORTED;
  if (T == 0 || B == 0) return SAKI_OK;
  if (!out || !aligned(out, 16) || !tables || !lens || !cu || !rows_ok(q, ld_q, H_q, dtype)) return SAKI_ERR_ARG;
  const ChunkPlan p = chunk_plan(dtype, T, B, G, H_kv, max_blocks);
  if (p.splits > 1 && (!ws || !aligned(ws, 16) || ws_bytes < p.ws_bytes())) return SAKI_ERR_WORKSPACE;
  const Chunk4Args a{q, ld_q, (const uint8_t*)k_cache, (const uint8_t*)v_cache, (const uint8_t*)scales, n_blocks,
                     tables, max_blocks, lens, cu, B, H_q, H_kv, T, out, p.splits};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == SAKI_F32) return p.halves ? launch_chunk<true, 2>(p, a, ws, s) : launch_chunk<true, 1>(p, a, ws, s);
  return p.halves ? launch_chunk<false, 2>(p, a, ws, s) : launch_chunk<false, 1>(p, a, ws, s);
}

}  // extern "C"
