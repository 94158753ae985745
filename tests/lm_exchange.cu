// Drives the exchange of a cluster's maps (csrc/lm_glr.h) with a block that stops sending: a cluster of two
// blocks, of which the second takes part in `sent` rounds and then goes to the last barrier.  Every wait is
// bounded; the first block records each round's state before a thread's chunk and after the round.
#include "lm_glr.h"

using namespace gem::lm;
using namespace gem::lm::glr;

constexpr int kThreads = 64, kBlocks = 2;

template <int V>
__global__ void __launch_bounds__(kThreads) exchange_kernel(float* out, int rounds, int sent, int first_reset) {
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  __shared__ __align__(16) Map<V> blocks[2 * kBlocks * 32];   // (a map of two channels is sent as one 16-byte store)
  __shared__ Exchange exchange;
  start_exchange<true>(exchange);
  const int rank = blockIdx.x % kBlocks;
  Vec<V> state = splat<V>(1.0f);
  for (int round = 0; round < (rank == 0 ? rounds : sent); ++round) {
    const Map<V> own = {splat<V>(round >= first_reset ? -1.0f : 0.5f), splat<V>(1.0f)};
    const Vec<V> before = scan_round<V, true, true>(own, round, kThreads / 32, rank, kBlocks, maps, blocks, exchange, state);
    if (rank == 0)
      for (int v = 0; v < V; ++v) {
        out[((round * kThreads + threadIdx.x) * 2 + 0) * V + v] = before.v[v];
        out[((round * kThreads + threadIdx.x) * 2 + 1) * V + v] = state.v[v];
      }
  }
  cg::this_cluster().sync();
}

template <int V>
static int run(float* out, int rounds, int sent, int first_reset) {
  const cudaError_t e = launch_cluster_pdl(&exchange_kernel<V>, unsigned(kBlocks), unsigned(kThreads), unsigned(kBlocks), 0, nullptr, out,
                                           rounds, sent, first_reset);
  return e != cudaSuccess ? int(e) : int(cudaDeviceSynchronize());
}

extern "C" int run_exchange(int channels, float* out, int rounds, int sent, int first_reset) {
  return channels == 2 ? run<2>(out, rounds, sent, first_reset) : run<1>(out, rounds, sent, first_reset);
}
