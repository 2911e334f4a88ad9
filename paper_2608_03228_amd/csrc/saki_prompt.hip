// Causal attention of whole prompts for gfx950 (CDNA4, wave64):
//
//   prompt_attend_kernel  bf16, on the 32x32x16 MFMA
//   prompt_attend_f32_kernel  float32, on the 32x32x2 MFMA

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>

#include "saki.h"
#include "saki_internal.h"
#include "saki_topk.h"

namespace {

using saki::kHeadDim;
using saki_dev::kWave;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kScale = 0.08838834764831845f;  // 1 / sqrt(d)
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kRows = 128;    // query rows of a work-group (32 a wave)
constexpr int kKeys = 64;     // keys of a tile

struct PromptArgs {
  const void *q, *k, *v;
  size_t ld_q, ld_k, ld_v;  // elements between tokens
  const int* cu;
  int B, H_q, H_kv, T;
  void* out;
  int tiles;  // row blocks of all prompts, at most
};

// Row block `x` of the packed prompts.  The rows of one KV head are (token,
// query head of its group) pairs, token after token; a prompt's blocks of
// kRows rows start at floor(first row / kRows) + b, which leaves each prompt
// its own ones (with gaps), so that a block finds its prompt by bisection.
struct Block {
  int b, start, len, row0;  // prompt, its first token and length, first row in it; len = 0: none
};
__device__ __forceinline__ Block find_block(const PromptArgs& a, int x) {
  const int G = a.H_q / a.H_kv;
  auto at = [&](int b) { return min(max(a.cu[b], 0), a.T); };
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((long long)at(mid) * G / kRows + mid <= x)
      lo = mid;
    else
      hi = mid;
  }
  Block r;
  r.b = lo;
  r.start = at(lo);
  r.len = max(at(lo + 1) - r.start, 0);
  const long long row0 = (x - ((long long)r.start * G / kRows + lo)) * kRows;
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

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

__global__ __launch_bounds__(256, 2) void prompt_attend_kernel(PromptArgs a) {
  __shared__ alignas(1024) uint8_t lds[2][2][kKeys * kHeadDim * 2];  // [buffer][keys, values]
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int hk = blockIdx.x % a.H_kv, G = a.H_q / a.H_kv;
  const Block blk = find_block(a, a.tiles - 1 - (int)(blockIdx.x / a.H_kv));
  if (blk.len == 0) return;
  const int n_rows = (int)min((long long)blk.len * G - blk.row0, (long long)kRows);
  const int n = lane % 32, h = lane / 32;

  // this lane's query row, its token and head
  const int row = min(wave * 32 + n, n_rows - 1) + blk.row0;
  const int pos = row / G;
  const size_t q_at = (size_t)(blk.start + pos) * a.ld_q + (size_t)(hk * G + row % G) * kHeadDim;
  bf16x8_t q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const uint4 v = *reinterpret_cast<const uint4*>((const __bf16*)a.q + q_at + 16 * s + 8 * h);
    __builtin_memcpy(&q[s], &v, 16);
  }
  const int pos_lo = (blk.row0 + min(wave * 32, n_rows - 1)) / G;
  const int pos_hi = (blk.row0 + min(wave * 32 + 31, n_rows - 1)) / G;
  const int n_tiles = (blk.row0 + n_rows - 1) / G / kKeys + 1;

  // staging: a wave's load takes 4 rows of 16 pieces; piece c of key row r goes
  // to place c ^ (r % 16) (keys), c ^ (r % 4 * 4) (values)
  const __bf16* kp = (const __bf16*)a.k + (size_t)blk.start * a.ld_k + (size_t)hk * kHeadDim;
  const __bf16* vp = (const __bf16*)a.v + (size_t)blk.start * a.ld_v + (size_t)hk * kHeadDim;
  auto stage = [&](int t, int buf) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = 16 * wave + 4 * u + lane / 16;
      const int tok = min(t * kKeys + r, blk.len - 1);
      const int ck = (lane % 16) ^ (r % 16), cv = (lane % 16) ^ (r % 4 * 4);
      __builtin_amdgcn_global_load_lds((global_void*)(kp + (size_t)tok * a.ld_k + ck * 8),
                                       (lds_void*)(lds[buf][0] + (16 * wave + 4 * u) * 256), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((global_void*)(vp + (size_t)tok * a.ld_v + cv * 8),
                                       (lds_void*)(lds[buf][1] + (16 * wave + 4 * u) * 256), 16, 0, 0);
    }
  };

  f32x16_t o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int k_lane = n * 256 + ((h ^ (lane % 16)) * 16);
  const int vs = lane % 16, vg = lane / 16;
  const int v_lane = (4 * (vg / 2) + vs / 4) * 256 + 32 * (vg % 2) + 8 * (vs % 4);

  stage(0, 0);
  for (int t = 0; t < n_tiles; ++t) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's part of tile t
    __syncthreads();
    if (t + 1 < n_tiles) stage(t + 1, (t + 1) & 1);
    if (t * kKeys > pos_hi) continue;
    const uint8_t *kt = lds[t & 1][0], *vt = lds[t & 1][1];
    f32x16_t s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        bf16x8_t kf;
        __builtin_memcpy(&kf, kt + b * 32 * 256 + (k_lane ^ (x * 32)), 16);
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[x], s[b], 0, 0, 0);
      }
    }
    if (t * kKeys + kKeys - 1 > pos_lo) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t * kKeys + 32 * b + 8 * (i / 4) + 4 * h + i % 4 > pos) s[b][i] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[1][i]);
    top = fmaxf(top, swap32(top));
    if (__any(top > m)) {
      const float m1 = fmaxf(m, top);
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m1) * (kScale * kLog2e));
      m = m1;
      l *= keep;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= keep;
    }
    const float shift = -m * (kScale * kLog2e);
    uint32_t p[16];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], kScale * kLog2e, shift));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], kScale * kLog2e, shift));
        l += p0 + p1;
        p[8 * b + i / 2] = pack_bf16(p0, p1);
      }
#pragma unroll
    for (int x = 0; x < 4; ++x) {  // 16 keys each
      bf16x8_t pf;
      __builtin_memcpy(&pf, &p[4 * x], 16);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
        const uint8_t* at = vt + x * 16 * 256 + (v_lane ^ ((d ^ (vs / 4)) * 64));
        const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds_void*)at);
        const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds_void*)(at + 8 * 256));
        bf16x8_t vf;
        __builtin_memcpy(&vf, &lo, 8);
        __builtin_memcpy((char*)&vf + 8, &hi, 8);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[d], 0, 0, 0);
      }
    }
  }
  l += swap32(l);
  const float inv = 1.f / l;
  if (wave * 32 + n < n_rows) {
    __bf16* out = (__bf16*)a.out + ((size_t)(blk.start + pos) * a.H_q + hk * G + row % G) * kHeadDim;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<uint2*>(out + 32 * d + 2 * i + 4 * h) =
            make_uint2(pack_bf16(o[d][i] * inv, o[d][i + 1] * inv), pack_bf16(o[d][i + 2] * inv, o[d][i + 3] * inv));
  }
}

// float32: the same with every product on the float32 MFMA.  A work-group's
// waves hold their queries in LDS-free registers; keys and values are staged
// as rows of 128 floats.
constexpr int kKeysF32 = 32;
__global__ __launch_bounds__(256, 2) void prompt_attend_f32_kernel(PromptArgs a) {
  __shared__ alignas(16) float lds[2][2][kKeysF32][kHeadDim + 4];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int hk = blockIdx.x % a.H_kv, G = a.H_q / a.H_kv;
  const Block blk = find_block(a, a.tiles - 1 - (int)(blockIdx.x / a.H_kv));
  if (blk.len == 0) return;
  const int n_rows = (int)min((long long)blk.len * G - blk.row0, (long long)kRows);
  const int n = lane % 32, h = lane / 32;
  const int row = min(wave * 32 + n, n_rows - 1) + blk.row0;
  const int pos = row / G;
  const size_t q_at = (size_t)(blk.start + pos) * a.ld_q + (size_t)(hk * G + row % G) * kHeadDim;
  // dims 8 x + 4 h .. + 3 for x = 0 .. 15
  float4 q[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) q[x] = *reinterpret_cast<const float4*>((const float*)a.q + q_at + 8 * x + 4 * h);
  const int pos_lo = (blk.row0 + min(wave * 32, n_rows - 1)) / G;
  const int pos_hi = (blk.row0 + min(wave * 32 + 31, n_rows - 1)) / G;
  const int n_tiles = (blk.row0 + n_rows - 1) / G / kKeysF32 + 1;
  const float* kp = (const float*)a.k + (size_t)blk.start * a.ld_k + (size_t)hk * kHeadDim;
  const float* vp = (const float*)a.v + (size_t)blk.start * a.ld_v + (size_t)hk * kHeadDim;
  float4 kx[4], vx[4];
  const int sr = threadIdx.x / 32, sc = threadIdx.x % 32 * 4;
  auto load = [&](int t) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int tok = min(t * kKeysF32 + sr + 8 * u, blk.len - 1);
      kx[u] = *reinterpret_cast<const float4*>(kp + (size_t)tok * a.ld_k + sc);
      vx[u] = *reinterpret_cast<const float4*>(vp + (size_t)tok * a.ld_v + sc);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      *reinterpret_cast<float4*>(&lds[buf][0][sr + 8 * u][sc]) = kx[u];
      *reinterpret_cast<float4*>(&lds[buf][1][sr + 8 * u][sc]) = vx[u];
    }
  };
  f32x16_t o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  load(0);
  put(0);
  for (int t = 0; t < n_tiles; ++t) {
    __syncthreads();
    if (t + 1 < n_tiles) load(t + 1);
    if (t * kKeysF32 <= pos_hi) {
      const auto& kt = lds[t & 1][0];
      const auto& vt = lds[t & 1][1];
      f32x16_t s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float4 kf = *reinterpret_cast<const float4*>(&kt[n][8 * x + 4 * h]);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.x, q[x].x, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.y, q[x].y, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.z, q[x].z, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.w, q[x].w, s, 0, 0, 0);
      }
      if (t * kKeysF32 + kKeysF32 - 1 > pos_lo) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t * kKeysF32 + 8 * (i / 4) + 4 * h + i % 4 > pos) s[i] = -INFINITY;
      }
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      top = fmaxf(top, swap32(top));
      if (__any(top > m)) {
        const float m1 = fmaxf(m, top);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m1) * (kScale * kLog2e));
        m = m1;
        l *= keep;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= keep;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f((s[i] - m) * (kScale * kLog2e));
        l += s[i];
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vt[8 * (i / 4) + 4 * h + i % 4][32 * d + n], s[i], o[d], 0, 0, 0);
    }
    if (t + 1 < n_tiles) put((t + 1) & 1);
  }
  l += swap32(l);
  const float inv = 1.f / l;
  if (wave * 32 + n < n_rows) {
    float* out = (float*)a.out + ((size_t)(blk.start + pos) * a.H_q + hk * G + row % G) * kHeadDim;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(out + 32 * d + 2 * i + 4 * h) =
            make_float4(o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv);
  }
}

// Token rows of H heads at `p`, ld elements apart: what the 16-byte accesses need.
bool rows_ok(const void* p, size_t ld, int H, int dtype) {
  return p && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld >= (size_t)H * kHeadDim &&
         ld * (dtype == SAKI_F32 ? 4 : 2) % 16 == 0 && ld <= ((size_t)1 << 40);
}

}  // namespace

extern "C" {

int saki_attend_prompt(const void* q, const void* k, const void* v, int dtype, int T, int B, int H_q, int H_kv,
                       int d, size_t ld_q, size_t ld_k, size_t ld_v, const int* cu, void* out, void* stream) {
  if (T < 0 || B < 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || d <= 0) return SAKI_ERR_ARG;
  if (d != kHeadDim || (dtype != SAKI_F32 && dtype != SAKI_BF16)) return SAKI_ERR_UNSUPPORTED;
  // row numbers of a KV head fit an int, a launch's threads 32 bits
  const long long rows = (long long)T * (H_q / H_kv);
  const long long tiles = rows / kRows + B;
  if (rows > INT_MAX / 2 || B > INT_MAX / 2 || tiles * H_kv > (1 << 23)) return SAKI_ERR_UNSUPPORTED;
  if (T == 0 || B == 0) return SAKI_OK;
  if (!cu || !out || reinterpret_cast<uintptr_t>(out) % 16 || !rows_ok(q, ld_q, H_q, dtype) ||
      !rows_ok(k, ld_k, H_kv, dtype) || !rows_ok(v, ld_v, H_kv, dtype))
    return SAKI_ERR_ARG;
  const PromptArgs a{q, k, v, ld_q, ld_k, ld_v, cu, B, H_q, H_kv, T, out, (int)tiles};
  const dim3 grid((unsigned)(tiles * H_kv));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == SAKI_F32)
    hipLaunchKernelGGL(prompt_attend_f32_kernel, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(prompt_attend_kernel, grid, dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"
