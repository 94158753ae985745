// Embedding of tokens and the gradient of its table (include/gem_lm.h).
#include "lm_internal.h"

namespace gem {
namespace lm {
namespace {

constexpr int kEmbedThreads = 256;

struct EmbedArgs {
  const void* table;
  void* out;
  int64_t table_ld, out_ld;
  int64_t N;
  int V, D;
  const int32_t* tokens;
  float scale;
};

template <typename T, typename E>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs p) {
  pdl_entry();
  const int64_t n = blockIdx.x;
  const int token = p.tokens[n];
  const T* row = static_cast<const T*>(p.table) + int64_t(token) * p.table_ld;
  E* const out = static_cast<E*>(p.out) + n * p.out_ld;
  for (int d = threadIdx.x; d < p.D; d += kEmbedThreads)
    out[d] = from_f32<E>(token < 0 ? 0.0f : token >= p.V ? NAN : to_f32(row[d]) * p.scale);
}

struct EmbedGradArgs {
  const void* dout;
  void* dtable;
  int64_t dout_ld, dtable_ld;
  int64_t N;
  int V, D;
  const int32_t* tokens;
  float scale;
  int accumulate;
};

template <typename E, typename G>
__global__ void __launch_bounds__(kEmbedThreads) embed_grad_kernel(const EmbedGradArgs p) {
  pdl_entry();
  const int v = blockIdx.x;
  const int d = blockIdx.y * kEmbedThreads + threadIdx.x;
  float sum = 0.0f;
  bool any = false;
  for (int64_t n = 0; n < p.N; ++n)
    if (p.tokens[n] == v) {
      any = true;
      if (d < p.D) sum += to_f32(static_cast<const E*>(p.dout)[n * p.dout_ld + d]);
    }
  G* const out = static_cast<G*>(p.dtable) + v * p.dtable_ld + d;
  if (d >= p.D || (p.accumulate && !any)) return;
  *out = from_f32<G>(sum * p.scale + (p.accumulate ? to_f32(*out) : 0.0f));
}

constexpr int64_t kMaxTokens = int64_t(1) << 27, kMaxRowsOfTable = int64_t(1) << 30, kMaxWidth = int64_t(1) << 24;

bool embed_sizes_ok(int64_t N, int64_t V, int64_t D) {
  return N >= 0 && N <= kMaxTokens && V >= 1 && V <= kMaxRowsOfTable && D >= 0 && D <= kMaxWidth;
}
bool matrix_ok(const void* p, int dtype, int64_t D, int64_t ld) {
  return p && aligned_to(p, size_t(dtype_size(dtype))) && ld >= D && ld <= kMaxStride >> 16;
}

template <typename E, typename T>
cudaError_t launch_embed_as(const EmbedArgs& p, cudaStream_t stream) {
  return launch_pdl(embed_kernel<T, E>, dim3(unsigned(p.N)), dim3(kEmbedThreads), 0, stream, p);
}
template <typename T>
cudaError_t launch_embed(const EmbedArgs& p, int dtype, cudaStream_t stream) {
  return dtype == GEM_F32    ? launch_embed_as<float, T>(p, stream)
         : dtype == GEM_BF16 ? launch_embed_as<__nv_bfloat16, T>(p, stream)
                             : launch_embed_as<__half, T>(p, stream);
}

template <typename E, typename G>
cudaError_t launch_embed_grad_as(const EmbedGradArgs& p, cudaStream_t stream) {
  return launch_pdl(embed_grad_kernel<E, G>, dim3(unsigned(p.V), unsigned((p.D + kEmbedThreads - 1) / kEmbedThreads)),
                    dim3(kEmbedThreads), 0, stream, p);
}
template <typename E>
cudaError_t launch_embed_grad(const EmbedGradArgs& p, int grad_dtype, cudaStream_t stream) {
  return grad_dtype == GEM_F32    ? launch_embed_grad_as<E, float>(p, stream)
         : grad_dtype == GEM_BF16 ? launch_embed_grad_as<E, __nv_bfloat16>(p, stream)
                                  : launch_embed_grad_as<E, __half>(p, stream);
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

extern "C" {

int gem_embed(int table_dtype, int dtype, int64_t N, int64_t V, int64_t D, const void* table,
              int64_t table_ld, const int32_t* tokens, float scale, void* out, int64_t out_ld,
              void* stream) {
  if (!dtype_ok(table_dtype) || !dtype_ok(dtype) || !embed_sizes_ok(N, V, D)) return GEM_EINVAL;
  if (N == 0 || D == 0) return GEM_OK;
  if (!matrix_ok(table, table_dtype, D, table_ld) || !matrix_ok(out, dtype, D, out_ld) || !array_ok(tokens)) return GEM_EINVAL;
  const EmbedArgs p = {table, out, table_ld, out_ld, N, int(V), int(D), tokens, scale};
  const int as = dtype;
  dtype = table_dtype;
  return launch_status(BY_TYPE(launch_embed, p, as, static_cast<cudaStream_t>(stream)));
}

int64_t gem_embed_workspace(int64_t N, int64_t V, int64_t D) {
  if (!embed_sizes_ok(N, V, D)) return -1;
  return 16 * N;
}

int gem_embed_grad(int dtype, int grad_dtype, int64_t N, int64_t V, int64_t D, const void* dout,
                   int64_t dout_ld, const int32_t* tokens, float scale, int accumulate,
                   void* dtable, int64_t dtable_ld, void* workspace, void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(grad_dtype) || !embed_sizes_ok(N, V, D) || (accumulate & ~1)) return GEM_EINVAL;
  if (D == 0 || (N == 0 && accumulate)) return GEM_OK;
  if (!matrix_ok(dtable, grad_dtype, D, dtable_ld)) return GEM_EINVAL;
  if (N > 0 && (!matrix_ok(dout, dtype, D, dout_ld) || !array_ok(tokens))) return GEM_EINVAL;
  if (N > 0 && (!workspace || !aligned_to(workspace, 16))) return GEM_EINVAL;
  const EmbedGradArgs p = {dout, dtable, dout_ld, dtable_ld, N, int(V), int(D), tokens, scale, accumulate};
  return launch_status(BY_TYPE(launch_embed_grad, p, grad_dtype, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
