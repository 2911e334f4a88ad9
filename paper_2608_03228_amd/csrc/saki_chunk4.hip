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
constexpr int kRows = 128;                      // query rows of a work-group (32 a wave)
// A row's sums are scaled down only once a score passes the maximum they go by
// by this many powers of two.
constexpr float kSlack = 8.f;
constexpr size_t kChunkPart = (size_t)kRows * (kHeadDim + 2);  // floats of a part: sums, maxima, weights

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
// multiplied.  S^T = K Q^T leaves a lane with scores of one row, so the softmax is
// in registers but for one exchange, and its weights are at once the operand of
// O^T = V^T P^T, whose other operand the transposing LDS reads form.  bf16: weights
// rounded to bf16; float32: queries and weights in three bf16 terms, 32 keys at a
// time for the registers' sake.
template <bool F32, bool SPLIT>
__global__ __launch_bounds__(256, 2) void cache4_prompt_kernel(Chunk4Args a, float* __restrict__ ws) {
  using T = std::conditional_t<F32, float, __bf16>;
  constexpr int kQT = F32 ? 3 : 1;
  constexpr int NB = F32 ? 1 : 2;  // 32 keys each, between two looks at the maximum
  constexpr int kTileBytes = kTile * kHeadDim * 2;
  // two arrays, and the loop below unrolled over them: a read of one is then known
  // not to meet the writes to the other
  __shared__ alignas(1024) uint8_t lds_a[2 * kTileBytes], lds_b[2 * kTileBytes];  // keys, values
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int hk = blockIdx.x % a.H_kv, G = a.H_q / a.H_kv;
  const int part = blockIdx.x / a.H_kv, sp = SPLIT ? part % a.splits : 0, x = SPLIT ? part / a.splits : part;
  const Block blk = saki_dev::find_block(a.cu, a.B, a.T, x, G, kRows);
  if (blk.len == 0) return;
  const int n_rows = (int)min((long long)blk.len * G - blk.row0, (long long)kRows);
  const int n = lane % 32, h = lane / 32, rw = wave * 32;

  // this lane's row, its token, head and position; the least and largest position
  // of the group's rows and of the wave's
  const int row = min(rw + n, n_rows - 1) + blk.row0, tok = row / G;
  const int before = a.lens[blk.b] - blk.len;
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

  const int* table = a.tables + (size_t)blk.b * a.max_blocks;
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
      *reinterpret_cast<uint4*>(to + r * 256 + (((tid % 4 * 4 + s) ^ (r % 16)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float f = __uint_as_float(__builtin_amdgcn_alignbit(ve[c], ve[c], turn) & 0x7f800000u);
      // a weight of zero has to make them zero: tokens that no row sees, and NaN where a row may not see it (below)
      const int u = t * kTile + v0 + c;
      if (u > pos_max || (u > pos_min && __float_as_uint(f) == 0x7f800000u)) f = 0.f;
      uint32_t w[4];
      decode8(vc[c], f, w);
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
    for (int b0 = 0; b0 < 2; b0 += NB) {
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
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m1) * (kScale * kLog2e));
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

  int at0 = block_of(t0), at1 = block_of(t0 + 1);
  fetch(at0);
  if (at0 >= 0) put(t0, lds_a);
  fetch(at1);
  auto step = [&](int t, const uint8_t* now, uint8_t* next) __attribute__((always_inline)) {
    __syncthreads();  // block t is in `now`, and `next` is read
    const int at2 = block_of(t + 2);
    if (at1 >= 0) put(t + 1, next);
    fetch(at2);
    if (at0 >= 0) tile(t, now);
    at0 = at1;
    at1 = at2;
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
  if (rw + n >= n_rows) return;
  if constexpr (SPLIT) {
    float* w = ws + ((size_t)(x * a.H_kv + hk) * a.splits + sp) * kChunkPart;
    if (h == 0) w[kRows * kHeadDim + rw + n] = m, w[kRows * (kHeadDim + 1) + rw + n] = l;
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

// Joins a row block's parts: 8 threads a row, 16 dims each.
template <bool F32>
__global__ __launch_bounds__(256) void cache4_gather_kernel(Chunk4Args a, const float* __restrict__ ws) {
  using T = std::conditional_t<F32, float, __bf16>;
  const int hk = blockIdx.x % a.H_kv, x = blockIdx.x / a.H_kv, G = a.H_q / a.H_kv;
  const Block blk = saki_dev::find_block(a.cu, a.B, a.T, x, G, kRows);
  if (blk.len == 0) return;
  const int i = blockIdx.y * 32 + threadIdx.x / 8, d0 = threadIdx.x % 8 * 16;
  if (i >= (long long)blk.len * G - blk.row0) return;
  const float* w = ws + (size_t)(x * a.H_kv + hk) * a.splits * kChunkPart;
  float M = -INFINITY, L = 0.f, y[16];
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, w[s * kChunkPart + kRows * kHeadDim + i]);
  const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float* p = w + s * kChunkPart;
    const float l = p[kRows * (kHeadDim + 1) + i];
    if (l == 0.f) continue;  // no key of the part is seen (a NaN goes on)
    const float f = __builtin_amdgcn_exp2f((p[kRows * kHeadDim + i] - ref) * (kScale * kLog2e));
    float z[16];
    load_elems<float, 16>(p + (size_t)i * kHeadDim + d0, z);
    L += l * f;
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] += z[e] * f;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] *= inv;
  const int row = blk.row0 + i;
  store_elems<T, 16>((T*)a.out + ((size_t)(blk.start + row / G) * a.H_q + hk * G + row % G) * kHeadDim + d0, y);
}

// Row blocks of the packed tokens, at most.
long long chunk_blocks(int T, int B, int G) { return (long long)T * G / kRows + B; }

// Work-groups that share a row block's keys: as many as fill the GPU, two a CU,
// with at least four cache blocks each.
int chunk_splits(long long groups, int max_blocks) {
  long long s = 512 / groups;
  const long long most = max_blocks / 4;
  s = s > most ? most : s;
  return (int)(s < 1 ? 1 : s);
}

}  // namespace

extern "C" {

size_t saki_cache4_prompt_workspace_bytes(int T, int B, int H_q, int H_kv, int max_blocks) {
  if (T < 0 || B < 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || max_blocks <= 0) return 0;
  if (T == 0 || B == 0) return 256;
  const long long groups = chunk_blocks(T, B, H_q / H_kv) * H_kv;
  const int splits = chunk_splits(groups, max_blocks);
  return splits > 1 ? (size_t)groups * splits * kChunkPart * sizeof(float) : 256;
}

int saki_cache4_prompt(const void* q, int dtype, int T, int B, int H_q, int H_kv, int d, size_t ld_q,
                       const void* k_cache, const void* v_cache, const void* scales, int n_blocks, const int* tables,
                       int max_blocks, const int* lens, const int* cu, void* out, void* ws, size_t ws_bytes,
                       void* stream) {
  if (T < 0 || B < 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || d <= 0 || max_blocks <= 0) return SAKI_ERR_ARG;
  const int st = check_cache4(k_cache, v_cache, scales, n_blocks, H_kv);
  if (st != SAKI_OK) return st;
  const int G = H_q / H_kv;
  const long long groups = chunk_blocks(T, B, G) * H_kv;
  if (d != kHeadDim || !type_ok(dtype) || T > kMaxTokens || max_blocks > INT_MAX / kTile - 1 ||
      (long long)T * G >= INT_MAX || groups > (1 << 23) || H_q > 65535)
    return SAKI_ERR_UNSUPPORTED;
  if (T == 0 || B == 0) return SAKI_OK;
  if (!out || !aligned(out, 16) || !tables || !lens || !cu || !rows_ok(q, ld_q, H_q, dtype)) return SAKI_ERR_ARG;
  const int splits = chunk_splits(groups, max_blocks);
  if (splits > 1 && (!ws || !aligned(ws, 16) || ws_bytes < saki_cache4_prompt_workspace_bytes(T, B, H_q, H_kv, max_blocks)))
    return SAKI_ERR_WORKSPACE;
  const Chunk4Args a{q, ld_q, (const uint8_t*)k_cache, (const uint8_t*)v_cache, (const uint8_t*)scales, n_blocks,
                     tables, max_blocks, lens, cu, B, H_q, H_kv, T, out, splits};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)(groups * splits)), join((unsigned)groups, kRows / 32);
  if (splits == 1) {
    if (dtype == SAKI_F32)
      hipLaunchKernelGGL((cache4_prompt_kernel<true, false>), grid, dim3(256), 0, s, a, nullptr);
    else
      hipLaunchKernelGGL((cache4_prompt_kernel<false, false>), grid, dim3(256), 0, s, a, nullptr);
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  if (dtype == SAKI_F32) {
    hipLaunchKernelGGL((cache4_prompt_kernel<true, true>), grid, dim3(256), 0, s, a, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    hipLaunchKernelGGL((cache4_gather_kernel<true>), join, dim3(256), 0, s, a, (const float*)ws);
  } else {
    hipLaunchKernelGGL((cache4_prompt_kernel<false, true>), grid, dim3(256), 0, s, a, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    hipLaunchKernelGGL((cache4_gather_kernel<false>), join, dim3(256), 0, s, a, (const float*)ws);
  }
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"
