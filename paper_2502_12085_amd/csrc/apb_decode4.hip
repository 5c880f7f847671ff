// Decoding-stage attention over a KV cache in 4 bits (the format of
// apb_cache4.hip), for gfx950.
//
// A workgroup owns one row (query head, new token) and walks the rows of the
// cache that it sees 256 at a time: a thread forms one key's logit, the workgroup the
// chunk's maximum and sum (online softmax in base 2, scale * log2(e) folded in), and
// a thread of each element of the head the value product.  Everything in fp32.
#include <math.h>

#include "apb_internal.h"

namespace apb {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float value4(unsigned code) {
  const unsigned m = code & 7;
  const float x = m < 2 ? 0.5f * (float)m : (float)(2 + (m & 1)) * (float)(1u << ((m >> 1) - 1)) * 0.5f;
  return code & 8 ? -x : x;
}

__device__ __forceinline__ float scale4(unsigned b) {
  return b == 255 ? NAN : __uint_as_float(b << 23);
}

template <int D>
__global__ void __launch_bounds__(kThreads) decode4_simple_kernel(Decode4Args a) {
  __shared__ float qs[D], p[kThreads], red[kThreads / 64], acc2[kThreads];
  const int tid = threadIdx.x;
  const int row = blockIdx.x;  // query head * n_new + token
  const int head = row / a.n_new, tok = row % a.n_new, kvh = head / (a.n_q / a.n_kv);
  const int vis = a.causal ? a.Lc - a.n_new + tok + 1 : a.Lc;
  const size_t base = (size_t)kvh * a.capacity;
  if (tid < D) qs[tid] = __uint_as_float((unsigned)a.q[(size_t)row * D + tid] << 16);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  constexpr int PARTS = kThreads / D;  // threads of one output element
  const int el = tid % D, part = tid / D;
  for (int c0 = 0; c0 < vis; c0 += kThreads) {
    const int c = c0 + tid;
    float s = -INFINITY;
    if (c < vis) {
      s = 0.f;
      for (int g = 0; g < D / 32; ++g) {
        float t = 0.f;
        for (int j = 0; j < 16; ++j) {
          const unsigned x = a.k_codes[(base + c) * (D / 2) + 16 * g + j];
          t = fmaf(value4(x & 15), qs[32 * g + 2 * j], t);
          t = fmaf(value4(x >> 4), qs[32 * g + 2 * j + 1], t);
        }
        s = fmaf(t, scale4(a.k_scales[(base + c) * (D / 32) + g]), s);
      }
      s *= a.scale_log2;
    }
    float mx = s;
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    if (tid % 64 == 0) red[tid / 64] = mx;
    __syncthreads();
    mx = m;
    for (int w = 0; w < kThreads / 64; ++w) mx = fmaxf(mx, red[w]);
    // (a NaN logit is no maximum; with no other its row stays at -inf and gets NaN)
    const float alpha = m == mx ? 1.f : exp2f(m - mx);
    const float e = s == -INFINITY ? 0.f : exp2f(s - mx);
    m = mx;
    p[tid] = e;
    float sum = e;
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    __syncthreads();
    if (tid % 64 == 0) red[tid / 64] = sum;
    __syncthreads();
    l *= alpha;
    for (int w = 0; w < kThreads / 64; ++w) l += red[w];
    o *= alpha;
    const int n = min(kThreads, vis - c0);
    for (int i = part; i < n; i += PARTS) {
      const size_t r = base + c0 + i;
      const unsigned x = a.v_codes[r * (D / 2) + el / 2] >> (4 * (el & 1)) & 15;
      o = fmaf(p[i], value4(x) * scale4(a.v_scales[r * (D / 32) + el / 32]), o);
    }
    __syncthreads();
  }
  acc2[tid] = o;
  __syncthreads();
  if (tid < D) {
    for (int q = 1; q < PARTS; ++q) o += acc2[q * D + tid];
    a.o[(size_t)row * D + tid] = vis > 0 ? o / l : 0.f;
    if (tid == 0) a.lse[row] = vis > 0 ? 0.69314718055994531f * (m + log2f(l)) : -INFINITY;
  }
}

}  // namespace

uint64_t decode4_workspace_bytes(const Decode4Args& a) {
  return (uint64_t)a.n_q * a.n_new * (a.head_dim + 1) * 4;
}

hipError_t launch_decode4(const Decode4Args& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.n_q * a.n_new));
  if (a.head_dim == 128) hipLaunchKernelGGL((decode4_simple_kernel<128>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((decode4_simple_kernel<64>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace apb
