// Attention over the paged 4-bit cache (include/laq_fp4.h: laq_fp4_attention).
//
// One wave per (token, query head): 64 rows at a time, a row's logit per lane, one pass with the running maximum and sum, then every lane
// sums its channels of V.
#include "laq_fp4_codes.h"

namespace laq {

namespace {

// Code c as fp32.
__device__ __forceinline__ float fp4_value(uint32_t c) {
  const uint32_t m = c & 7;
  const float x = m < 2 ? 0.5f * m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1) << 22);
  return c & 8 ? -x : x;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void put_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_value(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T>
__global__ __launch_bounds__(64) void fp4_attention_kernel(Fp4View c, Fp4Attention a) {
  __shared__ float qs[256];
  const int token = blockIdx.x, head = blockIdx.y, kv = head / (a.Hq / c.Hkv), lane = threadIdx.x;
  int inst = token, T_i = 1, t = 0;
  if (a.start) {
    if (token >= a.start[a.n]) return;
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.start[mid] <= token) lo = mid; else hi = mid;
    }
    inst = lo;
    T_i = a.start[lo + 1] - a.start[lo];
    t = token - a.start[lo];
  }
  const long long held = min((long long)max(a.rows[inst], 0), (long long)a.blocks_per_inst * c.block_rows);
  const int seen = (int)max(held - T_i + t + 1, 0ll);
  const T* q = static_cast<const T*>(a.q) + token * a.stride_token + head * a.stride_head;
  for (int i = lane; i < c.d; i += 64) qs[i] = to_float(q[i]);
  __syncthreads();
  float m = -INFINITY, z = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < seen; j0 += 64) {
    const int j = j0 + lane;
    float s = -INFINITY;
    int64_t codes = -1, scales = 0;
    if (j < seen) {
      const int b = a.table[(size_t)inst * a.blocks_per_inst + j / c.block_rows], r = j % c.block_rows;
      if (b >= 0 && b < c.n_blocks) {
        codes = b * c.block + kv * c.head + r * c.row;
        scales = b * c.scale_block + kv * c.scale_head + r * c.scale_row;
        float dot = 0.f;
        for (int i = 0; i < c.d; i += 2) {
          const uint32_t byte = c.k.codes[codes + i / 2], e = c.k.scales[scales + i / 32];
          const float scale = e == 255 ? NAN : fp4_scale_value(e);
          dot = fmaf(qs[i], fp4_value(byte & 15) * scale, dot);
          dot = fmaf(qs[i + 1], fp4_value(byte >> 4) * scale, dot);
        }
        s = dot * a.scale2;
      }
    }
    float top = s;
    for (int w = 1; w < 64; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
    const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
    const float p = codes >= 0 ? __builtin_amdgcn_exp2f(s - ref) : 0.f, w_old = __builtin_amdgcn_exp2f(m - ref);
    float sum = p;
    for (int w = 1; w < 64; w *= 2) sum += __shfl_xor(sum, w);
    z = z * w_old + sum;
    m = m_new;
    for (int i = 0; i < 4; ++i) o[i] *= w_old;
    for (int r = 0; r < 64; ++r) {
      const int64_t at = __shfl(codes, r), sc = __shfl(scales, r);
      const float w = __shfl(p, r);
      if (at < 0) continue;
      for (int i = 0; i < 4; ++i) {
        const int ch = lane + 64 * i;
        if (ch >= c.d) break;
        const uint32_t byte = c.v.codes[at + ch / 2], e = c.v.scales[sc + ch / 32];
        o[i] = fmaf(w, fp4_value(ch & 1 ? byte >> 4 : byte & 15) * (e == 255 ? NAN : fp4_scale_value(e)), o[i]);
      }
    }
  }
  for (int i = 0; i < 4; ++i) {
    const int ch = lane + 64 * i;
    if (ch < c.d) put_value(static_cast<T*>(a.out) + ((size_t)token * a.Hq + head) * c.d + ch, z == 0.f ? 0.f : o[i] / z);
  }
  if (a.lse && lane == 0) a.lse[(size_t)token * a.Hq + head] = z == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(z)) * 0.69314718055994530942f;
}

}  // namespace

size_t fp4_attention_bytes(const Fp4View&, int, int, int, int64_t, int) { return 0; }

hipError_t launch_fp4_attention(const Fp4View& c, int dtype, const Fp4Attention& a, void*, size_t, hipStream_t st) {
  const dim3 grid((unsigned)a.n_tokens, a.Hq);
  if (dtype == LAQ_BF16) hipLaunchKernelGGL(fp4_attention_kernel<uint16_t>, grid, dim3(64), 0, st, c, a);
  else hipLaunchKernelGGL(fp4_attention_kernel<float>, grid, dim3(64), 0, st, c, a);
  return hipGetLastError();
}

}  // namespace laq
