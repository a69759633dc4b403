// Log probabilities of given tokens, entropies, top alternatives (pb_log_probs) and their gradient (pb_log_probs_backward).
#include <math.h>

#include "pb_ops.h"

namespace pb {

constexpr int LB = 256;   // threads per workgroup

// Order of the alternatives: a larger key is a better one.  High half: the logit as an unsigned number that rises with it (both
// zeros the same, a NaN above all), low half: the index, lower ones first.  0 and all ones are no keys.
__device__ __forceinline__ uint64_t top_key(float x, uint32_t i) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = x != x ? 0xFFFFFFFEu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return (uint64_t)o << 32 | (uint32_t)~i;
}

template <class T, class OP>
__device__ T reduce(T x, T* lds, OP op) {
  lds[threadIdx.x] = x;
  __syncthreads();
  for (int s = LB / 2; s > 0; s >>= 1) {
    if ((int)threadIdx.x < s) lds[threadIdx.x] = op(lds[threadIdx.x], lds[threadIdx.x + s]);
    __syncthreads();
  }
  const T r = lds[0];
  __syncthreads();
  return r;
}

template <class T, class ID>
__global__ void __launch_bounds__(LB) k_logp(const LogpArgs a) {
  __shared__ float f[LB];
  __shared__ uint64_t u[LB];
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.logits + r * a.stride;
  float m = -INFINITY;
  for (int64_t j = threadIdx.x; j < a.vocab; j += LB) m = fmaxf(m, to_float(x[j]) * a.scale);
  m = reduce(m, f, [](float p, float q) { return fmaxf(p, q); });
  const float ref = m == -INFINITY ? 0.f : m;
  float s = 0.f, h = 0.f;
  for (int64_t j = threadIdx.x; j < a.vocab; j += LB) {
    const float d = to_float(x[j]) * a.scale - ref, e = expf(d);
    s += e;
    h += e * fmaxf(d, -150.f);
  }
  s = reduce(s, f, [](float p, float q) { return p + q; });
  h = reduce(h, f, [](float p, float q) { return p + q; });
  const bool empty = m == -INFINITY && s == 0.f;
  const float ls = empty ? 0.f : logf(s);
  if (threadIdx.x == 0) {
    a.norm[2 * r] = s != s ? s : m;
    a.norm[2 * r + 1] = ls;
    if (a.entropy) a.entropy[r] = empty ? 0.f : ls - h / s;
    if (a.logp) {
      const int64_t t = ((const ID*)a.targets)[r];
      a.logp[r] = t >= 0 && t < a.vocab ? to_float(x[t]) * a.scale - ref - ls : 0.f;
    }
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    uint64_t best = 0;
    for (int64_t j = threadIdx.x; j < a.vocab; j += LB) {
      const uint64_t key = top_key(to_float(x[j]), (uint32_t)j);
      if (key < last && key > best) best = key;
    }
    last = reduce(best, u, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
    if (threadIdx.x == 0) {
      const uint32_t j = ~(uint32_t)last;
      ((ID*)a.top_ids)[r * a.top + k] = (ID)j;
      a.top_logp[r * a.top + k] = to_float(x[j]) * a.scale - ref - ls;
    }
  }
}

template <class T, class ID>
__global__ void __launch_bounds__(LB) k_logp_grad(const LogpGradArgs a) {
  const int64_t r = blockIdx.y;
  for (int64_t row = r; row < a.rows; row += gridDim.y) {
    const T* x = (const T*)a.logits + row * a.stride;
    T* d = (T*)a.d + row * a.d_stride;
    const float m = a.norm[2 * row], ls = a.norm[2 * row + 1], ref = m == -INFINITY ? 0.f : m;
    const int64_t t = a.g_logp ? (int64_t)((const ID*)a.targets)[row] : -1;
    const float gl = t >= 0 && t < a.vocab ? a.g_logp[row] : 0.f;
    const float ge = a.g_entropy ? a.g_entropy[row] : 0.f, h = a.g_entropy ? a.entropy[row] : 0.f;
    for (int64_t j = (int64_t)blockIdx.x * LB + threadIdx.x; j < a.vocab; j += (int64_t)gridDim.x * LB) {
      const float ln = to_float(x[j]) * a.scale - ref - ls, p = expf(ln);
      float y = (j == t ? gl : 0.f) - gl * p;
      if (a.g_entropy) y -= ge * p * (fmaxf(ln, -150.f) + h);
      d[j] = from_float<T>(m == -INFINITY ? 0.f : y * a.scale);
    }
  }
}

int64_t logp_workspace(int64_t, int64_t, int) { return 0; }

void launch_logp(const LogpArgs& a, int dtype, int id_bits, hipStream_t s) {
  with_type(dtype, [&](auto t) { with_id(id_bits, [&](auto id) {
    hipLaunchKernelGGL((k_logp<decltype(t), decltype(id)>), dim3((unsigned)a.rows), dim3(LB), 0, s, a);
  }); });
}

void launch_logp_grad(const LogpGradArgs& a, int dtype, int id_bits, hipStream_t s) {
  const int64_t want = (a.vocab + 4 * LB - 1) / (4 * LB);
  const dim3 grid((unsigned)(want < 256 ? want : 256), (unsigned)(a.rows < 32768 ? a.rows : 32768));
  with_type(dtype, [&](auto t) { with_id(id_bits, [&](auto id) {
    hipLaunchKernelGGL((k_logp_grad<decltype(t), decltype(id)>), grid, dim3(LB), 0, s, a);
  }); });
}

}  // namespace pb
