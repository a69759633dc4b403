// Embedding lookup with a scale (pb_embed) and its gradient by sorted tokens (pb_embed_backward).
#include "pb_ops.h"

namespace pb {

constexpr int EB = 256;   // threads per workgroup

template <class T, class O, class ID>
__global__ void __launch_bounds__(EB) k_embed(const EmbedArgs a) {
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int64_t id = ((const ID*)a.ids)[i];
    const bool there = id >= 0 && id < a.vocab;
    const T* row = (const T*)a.table + (there ? id : 0) * a.dim;
    O* out = (O*)a.out + i * a.dim;
    for (int64_t j = threadIdx.x; j < a.dim; j += EB) out[j] = from_float<O>(there ? to_float(row[j]) * a.scale : 0.f);
  }
}

// ---- gradient: the places of the tokens sorted by id, equal ids in the order of their places, then the sum of each id's rows
__global__ void __launch_bounds__(EB) k_zero(uint32_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * EB + threadIdx.x; i < n; i += (int64_t)gridDim.x * EB) p[i] = 0;
}

template <class ID>
__global__ void __launch_bounds__(EB) k_count(const ID* ids, int64_t n, int64_t vocab, uint32_t* count) {
  for (int64_t i = (int64_t)blockIdx.x * EB + threadIdx.x; i < n; i += (int64_t)gridDim.x * EB) {
    const int64_t id = ids[i];
    if (id >= 0 && id < vocab) atomicAdd(count + id, 1u);
  }
}

// count -> the first place of each id among the sorted ones, one workgroup
__global__ void __launch_bounds__(EB) k_starts(uint32_t* count, int64_t vocab) {
  __shared__ uint32_t part[EB];
  const int64_t per = (vocab + EB - 1) / EB, lo = per * threadIdx.x, hi = lo + per < vocab ? lo + per : vocab;
  uint32_t s = 0;
  for (int64_t i = lo; i < hi; ++i) s += count[i];
  part[threadIdx.x] = s;
  __syncthreads();
  uint32_t at = 0;
  for (int i = 0; i < (int)threadIdx.x; ++i) at += part[i];
  for (int64_t i = lo; i < hi; ++i) {
    const uint32_t c = count[i];
    count[i] = at;
    at += c;
  }
}

// one workgroup takes the tokens in order, EB at a time; count[id] moves from the first place of the id to the one behind its last
template <class ID>
__global__ void __launch_bounds__(EB) k_place(const ID* ids, int64_t n, int64_t vocab, uint32_t* count, uint32_t* order) {
  __shared__ int64_t now[EB];
  for (int64_t base = 0; base < n; base += EB) {
    const int64_t i = base + threadIdx.x;
    int64_t id = i < n ? (int64_t)ids[i] : -1;
    if (id >= vocab) id = -1;
    now[threadIdx.x] = id;
    __syncthreads();
    uint32_t before = 0, behind = 0;
    for (int j = 0; j < EB; ++j) {
      if (now[j] != id) continue;
      before += j < (int)threadIdx.x;
      behind += j > (int)threadIdx.x;
    }
    uint32_t at = 0;
    if (id >= 0) {
      at = __hip_atomic_load(count + id, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + before;
      order[at] = (uint32_t)i;
    }
    __syncthreads();
    if (id >= 0 && behind == 0) __hip_atomic_store(count + id, at + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
  }
}

template <class T, class O>
__global__ void __launch_bounds__(EB) k_sum(const EmbedGradArgs a, const uint32_t* behind, const uint32_t* order) {
  for (int64_t v = blockIdx.x; v < a.vocab; v += gridDim.x) {
    const uint32_t lo = v ? behind[v - 1] : 0, hi = behind[v];
    if (lo == hi && a.add) continue;
    O* out = (O*)a.d_table + v * a.dim;
    for (int64_t j = threadIdx.x; j < a.dim; j += EB) {
      float s = 0.f;
      for (uint32_t k = lo; k < hi; ++k) s += to_float(((const T*)a.d_out)[(int64_t)order[k] * a.dim + j]);
      s *= a.scale;
      out[j] = from_float<O>(a.add ? to_float(out[j]) + s : s);
    }
  }
}

void launch_embed(const EmbedArgs& a, int dtype, int out_dtype, int id_bits, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n < (1 << 20) ? a.n : 1 << 20);
  with_type(dtype, [&](auto t) { with_type(out_dtype, [&](auto o) { with_id(id_bits, [&](auto id) {
    hipLaunchKernelGGL((k_embed<decltype(t), decltype(o), decltype(id)>), dim3(grid), dim3(EB), 0, s, a);
  }); }); });
}

int64_t embed_grad_workspace(int64_t n, int64_t vocab, int64_t) { return 4 * (n + vocab); }

void launch_embed_grad(const EmbedGradArgs& a, int dtype, int table_dtype, int id_bits, hipStream_t s) {
  uint32_t *count = (uint32_t*)a.workspace, *order = count + a.vocab;
  auto grid = [](int64_t n, int64_t most) { const int64_t g = (n + EB - 1) / EB; return dim3((unsigned)(g < most ? g : most)); };
  hipLaunchKernelGGL(k_zero, grid(a.vocab, 4096), dim3(EB), 0, s, count, a.vocab);
  if (a.n > 0) with_id(id_bits, [&](auto id) {
    using ID = decltype(id);
    hipLaunchKernelGGL((k_count<ID>), grid(a.n, 4096), dim3(EB), 0, s, (const ID*)a.ids, a.n, a.vocab, count);
    hipLaunchKernelGGL(k_starts, dim3(1), dim3(EB), 0, s, count, a.vocab);
    hipLaunchKernelGGL((k_place<ID>), dim3(1), dim3(EB), 0, s, (const ID*)a.ids, a.n, a.vocab, count, order);
  });
  with_type(dtype, [&](auto t) { with_type(table_dtype, [&](auto o) {
    hipLaunchKernelGGL((k_sum<decltype(t), decltype(o)>), dim3((unsigned)(a.vocab < (1 << 20) ? a.vocab : 1 << 20)), dim3(EB), 0, s, a, count, order);
  }); });
}

}  // namespace pb
