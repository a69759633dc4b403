// AdamW over many tensors at once, moments in 32 or in 8 bits (pb_adamw_step, pb_adamw_moments).
#include "pb_ops.h"

namespace pb {

// splitmix64's finaliser, as in the initial weights
__device__ __forceinline__ uint64_t mix(uint64_t z) {
  z ^= z >> 30; z *= 0xBF58476D1CE4E5B9ULL;
  z ^= z >> 27; z *= 0x94D049BB133111EBULL;
  return z ^ z >> 31;
}
constexpr uint64_t GOLDEN = 0x9E3779B97F4A7C15ULL;

// 8-bit moments.  With 3 bits kept behind the leading one, an fp32 number is its bit pattern >> 20 (exponent field and three
// bits), and a code counts these from the block's top downwards: encoding and decoding are integer shifts and sums.
constexpr int TOP_M = 15, TOP_V = 31;   // exponents below the block's that a code reaches: 4 bits of m's seven, 5 bits of v's eight
__device__ __forceinline__ int block_exponent(uint32_t largest) { return (int)((largest + (1u << 20)) >> 23); }
__device__ __forceinline__ float decode_m(uint32_t code, int e) {
  const int c = (int)(code & 127), q = c + 8 * (e - TOP_M);
  const float x = __uint_as_float(e == 255 ? 0x7FC00000u : c == 0 || q < 0 ? 0u : (uint32_t)q << 20);
  return code & 128 ? -x : x;
}
__device__ __forceinline__ float decode_v(uint32_t code, int e) {
  const int c = (int)code, q = c + 8 * (e - TOP_V);
  return __uint_as_float(e == 255 ? 0x7FC00000u : c == 0 || q < 0 ? 0u : (uint32_t)q << 20);
}
__device__ __forceinline__ uint32_t encode_m(float x, uint32_t dither, int e) {
  const uint32_t bits = __float_as_uint(x) & 0x7FFFFFFF;
  const int c = (int)((bits + dither) >> 20) - 8 * (e - TOP_M);
  return (bits == 0 || c < 0 ? 0u : c > 127 ? 127u : (uint32_t)c) | (x < 0.f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t encode_v(float x, uint32_t dither, int e) {
  const uint32_t bits = __float_as_uint(x);
  const int q = (int)((bits + dither) >> 20), c = (q < 1 ? 1 : q) - 8 * (e - TOP_V);
  return bits == 0 ? 0u : c < 1 ? 1u : c > 255 ? 255u : (uint32_t)c;
}

struct Coeffs { float lr, rs; };   // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
__device__ __forceinline__ double power(double x, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, x *= x)
    if (t & 1) r *= x;
  return r;
}
__device__ __forceinline__ Coeffs coeffs(const AdamWArgs& a, int64_t t) {
  if (t < 1) return {__uint_as_float(0x7FC00000u), 0.f};
  return {(float)(a.lr / (1.0 - power(a.beta1, t))), (float)(1.0 / sqrt(1.0 - power(a.beta2, t)))};
}

// The tensor a workgroup belongs to: a lane compares the first workgroup of a tensor of its own.
__device__ __forceinline__ int tensor_of(const AdamWArgs& a, int group) {
  const int lane = threadIdx.x & 63;
  const bool before = lane < a.n_tensors && a.first[lane < a.n_tensors ? lane : 0] <= group;
  return __builtin_amdgcn_readfirstlane((int)__popcll(__ballot(before)) - 1);
}

template <class W, class G, class H, int BITS>
__global__ void __launch_bounds__(ADAMW_CHUNK) k_adamw(const AdamWArgs a) {
  __shared__ uint32_t top[2][ADAMW_CHUNK];
  const int t = tensor_of(a, (int)blockIdx.x), tid = threadIdx.x;
  const int64_t i = (int64_t)((int)blockIdx.x - a.first[t]) * ADAMW_CHUNK + tid, at = a.at[t] + i;
  const int64_t step = a.step_dev ? *a.step_dev : a.step;
  const Coeffs k = coeffs(a, step);
  const bool mine = i < a.n[t];
  float m = 0.f, v = 0.f, g = 0.f, w = 0.f;
  if (mine) {
    g = to_float(((const G*)a.g[t])[i]);
    w = to_float(((const W*)a.w[t])[i]);
    if (a.grad_scale) g *= *a.grad_scale;
    if (BITS == 32) {
      m = ((const float*)a.m)[at];
      v = ((const float*)a.v)[at];
    } else {
      m = decode_m(((const uint8_t*)a.m)[at], a.m_exp[at / PB_ADAMW_BLOCK]);
      v = decode_v(((const uint8_t*)a.v)[at], a.v_exp[at / PB_ADAMW_BLOCK]);
    }
    // (each operation rounded: which code an 8-bit moment gets is defined by that)
    m = a.b1 * m + a.c1 * g;
    v = a.b2 * v + a.c2 * (g * g);
    const float d = k.lr * (m / (sqrtf(v) * k.rs + a.eps));
    w = w - a.decay[t] * w - d;
    ((W*)a.w[t])[i] = from_float<W>(w);
    if (a.hat[t]) ((H*)a.hat[t])[i] = from_float<H>(w - a.horizon * d);
  }
  if (BITS == 32) {
    if (mine) {
      ((float*)a.m)[at] = m;
      ((float*)a.v)[at] = v;
    }
    return;
  }
  top[0][tid] = __float_as_uint(m) & 0x7FFFFFFF;
  top[1][tid] = __float_as_uint(v) & 0x7FFFFFFF;
  __syncthreads();
  for (int s = ADAMW_CHUNK / 2; s > 0; s >>= 1) {
    if (tid < s) {
      top[0][tid] = max(top[0][tid], top[0][tid + s]);
      top[1][tid] = max(top[1][tid], top[1][tid + s]);
    }
    __syncthreads();
  }
  const int em = block_exponent(top[0][0]), ev = block_exponent(top[1][0]);
  const uint64_t key = mix(a.seed ^ mix((uint64_t)step));
  const uint64_t z = mix((uint64_t)(at >> 1) * GOLDEN + key) >> (at & 1 ? 32 : 0);
  ((uint8_t*)a.m)[at] = encode_m(m, (uint32_t)(z & 0xFFFF) << 4 | 8, em);
  ((uint8_t*)a.v)[at] = encode_v(v, (uint32_t)(z >> 16 & 0xFFFF) << 4 | 8, ev);
  if (tid == 0) {
    a.m_exp[at / PB_ADAMW_BLOCK] = (uint8_t)em;
    a.v_exp[at / PB_ADAMW_BLOCK] = (uint8_t)ev;
  }
}

__global__ void __launch_bounds__(256)
k_adamw_moments(const uint8_t* __restrict__ m, const uint8_t* __restrict__ v, const uint8_t* __restrict__ m_exp, const uint8_t* __restrict__ v_exp,
                int64_t n, float* __restrict__ m_out, float* __restrict__ v_out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    m_out[i] = decode_m(m[i], m_exp[i / PB_ADAMW_BLOCK]);
    v_out[i] = decode_v(v[i], v_exp[i / PB_ADAMW_BLOCK]);
  }
}

void launch_adamw(const AdamWArgs& a, int64_t groups, int w_type, int g_type, int hat_type, int bits, hipStream_t s) {
  with_type(w_type, [&](auto w) { with_type(g_type, [&](auto g) { with_type(hat_type, [&](auto h) {
    if (bits == 32) hipLaunchKernelGGL((k_adamw<decltype(w), decltype(g), decltype(h), 32>), dim3((unsigned)groups), dim3(ADAMW_CHUNK), 0, s, a);
    else hipLaunchKernelGGL((k_adamw<decltype(w), decltype(g), decltype(h), 8>), dim3((unsigned)groups), dim3(ADAMW_CHUNK), 0, s, a);
  }); }); });
}

void launch_adamw_moments(const uint8_t* m, const uint8_t* v, const uint8_t* m_exp, const uint8_t* v_exp, int64_t n, float* m_out, float* v_out, hipStream_t s) {
  const int64_t want = (n + 255) / 256;
  hipLaunchKernelGGL(k_adamw_moments, dim3((unsigned)(want < 8192 ? want : 8192)), dim3(256), 0, s, m, v, m_exp, v_exp, n, m_out, v_out);
}

}  // namespace pb
