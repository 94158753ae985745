// Short causal convolution of each channel over time (include/gem_lm.h).
//
// A thread has K neighbouring channels and walks over a segment of time with the last W inputs in
// registers, so x is read once but for the W - 1 steps before a segment.  The backward pass walks forward
// as well: step t's dp_t goes to the gradients of the W inputs it used, the oldest of which is then complete; it
// goes W - 1 steps past the segment for that.  Sums for the weights are taken in registers over the
// segment, in shared memory over the block's warps, and by a second kernel over the blocks, in that order.
#include "lm_internal.h"

namespace gem {
namespace lm {
namespace {

constexpr int kConvWarps = 4;       // most segments of time of a block, a warp each
constexpr int kSegment = 64;        // steps of a segment
constexpr int kAhead = 4;           // steps whose loads are in flight together
constexpr float kLog2e = 1.4426950408889634f;

struct ConvArgs {
  gem_seq_t x, y;          // backward: y is dx
  gem_seq_t dy;
  const float *weight, *bias, *state;
  float* state_last;
  const float* dstate_last;
  float* dstate;
  float* partial;          // [B blocks][W + 1][D]
  const int32_t* lengths;
  const uint8_t* reset;
  int64_t T;
  int D, columns, blocks;  // blocks along the channels, along a sequence's time
};

__device__ __forceinline__ float sigmoid(float v) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-v * kLog2e));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return r;
}

// K neighbouring elements as they are in memory (K = 1: any alignment, K = 4: aligned to all four).
template <typename E, int K>
struct alignas(sizeof(E) * K) Piece {
  E e[K];
};

// What a warp works on.
struct ConvPlace {
  int64_t b, first, end, n;   // its steps [first, end) of the sequence's n
  int64_t row;                // the block's number along sequences and time
  int d;                      // the thread's first channel
  bool on;
};
template <int K>
__device__ __forceinline__ ConvPlace conv_place(const ConvArgs& p) {
  ConvPlace a;
  a.row = blockIdx.x / p.columns;
  a.b = a.row / p.blocks;
  a.first = ((a.row % p.blocks) * (blockDim.x / 32) + threadIdx.x / 32) * kSegment;
  a.end = min(a.first + kSegment, p.T);
  a.n = p.lengths ? min(max(int64_t(p.lengths[a.b]), int64_t(0)), p.T) : p.T;
  a.d = ((blockIdx.x % p.columns) * 32 + threadIdx.x % 32) * K;
  a.on = a.d < p.D;
  return a;
}

template <int W, int K>
struct Taps {
  float w[W][K], bias[K];
  __device__ __forceinline__ void read(const ConvArgs& p, const ConvPlace& a) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      bias[k] = p.bias && a.on ? p.bias[a.d + k] : 0.0f;
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][k] = a.on ? p.weight[int64_t(a.d + k) * W + j] : 0.0f;
    }
  }
};

// The last W inputs, oldest first; tap j reaches W - 1 - j steps back, at most `age` of which lie in the
// step's own document.
template <typename E, int W, int K>
struct Window {
  float x[W][K];
  int age;

  // The inputs before the segment's first step (which lie in the sequence, or in its state).
  __device__ __forceinline__ void start(const ConvArgs& p, const ConvPlace& a, const E* row) {
    age = W;
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int k = 0; k < K; ++k) x[j][k] = 0.0f;
#pragma unroll
    for (int j = 1; j < W; ++j) {
      const int64_t t = a.first - W + j;
      if (t >= 0) {
        next(p, a, t);
        if (a.on) {
          const Piece<E, K> piece = *reinterpret_cast<const Piece<E, K>*>(row + t * p.x.stride_t);
#pragma unroll
          for (int k = 0; k < K; ++k) x[j][k] = to_f32(piece.e[k]);
        }
      } else if (p.state && a.on) {
#pragma unroll
        for (int k = 0; k < K; ++k) x[j][k] = p.state[(a.b * (W - 1) + t + W - 1) * p.D + a.d + k];
      }
    }
  }
  __device__ __forceinline__ void next(const ConvArgs& p, const ConvPlace& a, int64_t t) {
    age = p.reset && p.reset[a.b * p.T + t] ? 0 : min(age + 1, W);
  }
  __device__ __forceinline__ void push(const ConvArgs& p, const ConvPlace& a, int64_t t, const Piece<E, K>& piece) {
    next(p, a, t);
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
#pragma unroll
      for (int k = 0; k < K; ++k) x[j][k] = x[j + 1][k];
#pragma unroll
    for (int k = 0; k < K; ++k) x[W - 1][k] = to_f32(piece.e[k]);
    if (age < W - 1) {   // dropped inputs count as 0, whatever they hold
#pragma unroll
      for (int j = 0; j < W; ++j)
#pragma unroll
        for (int k = 0; k < K; ++k) x[j][k] = W - 1 - j > age ? 0.0f : x[j][k];
    }
  }
};

// The pieces of steps [t, t + kAhead) below `end` (zeros for a thread without channels).
template <typename E, int K>
__device__ __forceinline__ void read_ahead(Piece<E, K> (&to)[kAhead], const E* row, int64_t stride, int64_t t, int64_t end, bool on) {
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    to[u] = Piece<E, K>{};
    if (on && t + u < end) to[u] = *reinterpret_cast<const Piece<E, K>*>(row + (t + u) * stride);
  }
}
template <typename E, int K>
__device__ __forceinline__ void write_step(E* at, const float (&v)[K]) {
  Piece<E, K> piece;
#pragma unroll
  for (int k = 0; k < K; ++k) piece.e[k] = from_f32<E>(v[k]);
  *reinterpret_cast<Piece<E, K>*>(at) = piece;
}
template <typename E, int K>
__device__ __forceinline__ void write_zeros(E* row, int64_t stride, const ConvPlace& a) {
  if (!a.on) return;
  const float none[K] = {};
  for (int64_t t = max(a.first, a.n); t < a.end; ++t) write_step<E, K>(row + t * stride, none);
}

// A sequence's last inputs, by the warp whose segment it ends in (state_last may be state: only where one warp has
// the whole sequence, else conv_state_kernel writes them).
template <typename E, int W, int K, bool SILU>
__global__ void __launch_bounds__(kConvWarps * 32) conv_forward_kernel(const ConvArgs p) {
  pdl_entry();
  const ConvPlace a = conv_place<K>(p);
  const int64_t end = min(a.end, a.n);
  const E* const row = static_cast<const E*>(p.x.data) + a.b * p.x.stride_b + a.d;
  E* const out = static_cast<E*>(p.y.data) + a.b * p.y.stride_b + a.d;
  if (a.first < end || a.first == 0) {
    Taps<W, K> taps;
    taps.read(p, a);
    Window<E, W, K> win;
    win.start(p, a, row);
    Piece<E, K> ahead[kAhead], now[kAhead];
    read_ahead<E, K>(ahead, row, p.x.stride_t, a.first, end, a.on);
    for (int64_t t = a.first; t < end; t += kAhead) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) now[u] = ahead[u];
      read_ahead<E, K>(ahead, row, p.x.stride_t, t + kAhead, end, a.on);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (t + u >= end) break;
        win.push(p, a, t + u, now[u]);
        float y[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
          float v = taps.bias[k];
#pragma unroll
          for (int j = 0; j < W; ++j) v = fmaf(taps.w[j][k], win.x[j][k], v);
          y[k] = SILU ? v * sigmoid(v) : v;
        }
        if (a.on) write_step<E, K>(out + (t + u) * p.y.stride_t, y);
      }
    }
    if (p.state_last && a.on) {
#pragma unroll
      for (int j = 1; j < W; ++j)
#pragma unroll
        for (int k = 0; k < K; ++k) p.state_last[(a.b * (W - 1) + j - 1) * p.D + a.d + k] = win.x[j][k];
    }
  }
  write_zeros<E, K>(out, p.y.stride_t, a);
}

template <typename E, int W>
__global__ void __launch_bounds__(128) conv_state_kernel(const ConvArgs p, int64_t count) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * 128 + threadIdx.x;
  if (i >= count) return;
  const int64_t b = i / p.D, d = i % p.D;
  const int64_t n = p.lengths ? min(max(int64_t(p.lengths[b]), int64_t(0)), p.T) : p.T;
  float v[W - 1];
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) {
    const int64_t t = n - (W - 1) + j;
    v[j] = t >= 0  ? to_f32(static_cast<const E*>(p.x.data)[b * p.x.stride_b + t * p.x.stride_t + d])
           : p.state ? p.state[(b * (W - 1) + t + W - 1) * p.D + d]
                     : 0.0f;
    for (int64_t s = max(t + 1, int64_t(0)); p.reset && s < n; ++s)
      if (p.reset[b * p.T + s]) v[j] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) p.state_last[(b * (W - 1) + j) * p.D + d] = v[j];
}

template <typename E, int W, int K, bool SILU>
__global__ void __launch_bounds__(kConvWarps * 32) conv_backward_kernel(const ConvArgs p) {
  pdl_entry();
  __shared__ float sums[kConvWarps][W + 1][K][32];
  const ConvPlace a = conv_place<K>(p);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t end = min(a.end, a.n), reach = min(a.end + W - 1, a.n);
  const E* const row = static_cast<const E*>(p.x.data) + a.b * p.x.stride_b + a.d;
  const E* const dy = static_cast<const E*>(p.dy.data) + a.b * p.dy.stride_b + a.d;
  E* const out = static_cast<E*>(p.y.data) + a.b * p.y.stride_b + a.d;
  float dw[W + 1][K] = {};
  if (a.first < end || a.first == 0) {
    Taps<W, K> taps;
    taps.read(p, a);
    Window<E, W, K> win;
    win.start(p, a, row);
    float dx[W][K] = {};   // gradients of the window's inputs
    // the complete gradient of input t, which is the segment's, or the state's for the first one
    auto put = [&](int64_t t, const float (&v)[K]) {
      if (!a.on || t >= a.end) return;
      if (t >= a.first) {
        write_step<E, K>(out + t * p.y.stride_t, v);
      } else if (t < 0 && a.first == 0 && p.dstate) {
#pragma unroll
        for (int k = 0; k < K; ++k) p.dstate[(a.b * (W - 1) + t + W - 1) * p.D + a.d + k] = v[k];
      }
    };
    Piece<E, K> xs[kAhead], gs[kAhead], x_now[kAhead], g_now[kAhead];
    read_ahead<E, K>(xs, row, p.x.stride_t, a.first, reach, a.on);
    read_ahead<E, K>(gs, dy, p.dy.stride_t, a.first, reach, a.on);
    for (int64_t t0 = a.first; t0 < reach; t0 += kAhead) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        x_now[u] = xs[u];
        g_now[u] = gs[u];
      }
      read_ahead<E, K>(xs, row, p.x.stride_t, t0 + kAhead, reach, a.on);
      read_ahead<E, K>(gs, dy, p.dy.stride_t, t0 + kAhead, reach, a.on);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t t = t0 + u;
        if (t >= reach) break;
        win.push(p, a, t, x_now[u]);
        const bool own = t < end;   // (steps past the segment only complete its inputs' gradients)
#pragma unroll
        for (int k = 0; k < K; ++k) {
          float g = to_f32(g_now[u].e[k]);
          if (SILU) {
            float v = taps.bias[k];
#pragma unroll
            for (int j = 0; j < W; ++j) v = fmaf(taps.w[j][k], win.x[j][k], v);
            const float s = sigmoid(v);
            g *= s * fmaf(v, 1.0f - s, 1.0f);
          }
#pragma unroll
          for (int j = 0; j < W; ++j) {
            dx[j][k] = j + 1 < W ? dx[j + 1][k] : 0.0f;
            if (W - 1 - j <= win.age) dx[j][k] = fmaf(g, taps.w[j][k], dx[j][k]);
            if (own) dw[j][k] = fmaf(g, win.x[j][k], dw[j][k]);
          }
          if (own) dw[W][k] += g;
        }
        put(t - W + 1, dx[0]);
      }
    }
    if (reach == a.n) {   // the sequence ends here: no later step completes its last inputs
#pragma unroll
      for (int j = 1; j < W; ++j) {
        if (p.dstate_last && a.on && (a.n == 0 || W - 1 - j <= win.age)) {
#pragma unroll
          for (int k = 0; k < K; ++k) dx[j][k] += p.dstate_last[(a.b * (W - 1) + j - 1) * p.D + a.d + k];
        }
        put(a.n - W + j, dx[j]);
      }
    }
  }
  write_zeros<E, K>(out, p.y.stride_t, a);
  if (!p.partial) return;
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int k = 0; k < K; ++k) sums[warp][j][k][lane] = dw[j][k];
  __syncthreads();
  if (warp != 0 || !a.on) return;
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float v = dw[j][k];
      for (int q = 1; q < int(blockDim.x) / 32; ++q) v += sums[q][j][k][lane];
      p.partial[(a.row * (W + 1) + j) * p.D + a.d + k] = v;
    }
}

// Sums of the blocks' partial sums, a thread for each value.
__global__ void __launch_bounds__(128) conv_join_kernel(const float* partial, int64_t rows, int D, int W, float* dweight, float* dbias) {
  pdl_entry();
  const int d = blockIdx.x * 128 + threadIdx.x, j = blockIdx.y;
  if (d >= D) return;
  float v = 0.0f;
  for (int64_t i = 0; i < rows; ++i) v += partial[(i * (W + 1) + j) * D + d];
  if (j < W) {
    if (dweight) dweight[int64_t(d) * W + j] = v;
  } else if (dbias) {
    dbias[d] = v;
  }
}

// How time is cut: warps of a block, blocks of a sequence.
struct ConvCut {
  int64_t warps, blocks;
};
ConvCut conv_cut(int64_t T) {
  const int64_t segments = T < 1 ? 1 : (T + kSegment - 1) / kSegment, warps = segments < kConvWarps ? segments : kConvWarps;
  return {warps, (segments + warps - 1) / warps};
}

bool conv_sizes_ok(int64_t B, int64_t T, int64_t D, int W) {
  if (W < 2 || W > 4 || !extent_ok(B) || !extent_ok(T) || !extent_ok(D)) return false;
  const int64_t columns = (D + 31) / 32, blocks = conv_cut(T).blocks;
  return B == 0 || D == 0 || columns <= (kMaxExtent - 1) / blocks / B;   // a block at least for 32 channels and the steps of its warps
}

// Whether pieces of four channels of every step lie at multiples of their size.
bool in_fours(const gem_seq_t& s, int dtype, int64_t B, int64_t T, int64_t D) {
  return D % 4 == 0 && aligned_to(s.data, 4 * dtype_size(dtype)) && (B <= 1 || s.stride_b % 4 == 0) && (T <= 1 || s.stride_t % 4 == 0);
}

template <typename E, int W, int K>
cudaError_t launch_conv_as(ConvArgs p, int form, int64_t B, bool backward, cudaStream_t stream) {
  const ConvCut cut = conv_cut(p.T);
  const bool whole = p.T <= kSegment;   // a warp has the whole sequence
  float* const state_last = p.state_last;
  if (!whole) p.state_last = nullptr;
  p.columns = (p.D + 32 * K - 1) / (32 * K);
  p.blocks = int(cut.blocks);
  const dim3 grid(unsigned(B * p.blocks * p.columns)), block(unsigned(cut.warps * 32));
  const bool silu = form == GEM_CONV_SILU;
  if (backward)
    return silu ? launch_pdl(conv_backward_kernel<E, W, K, true>, grid, block, 0, stream, p)
                : launch_pdl(conv_backward_kernel<E, W, K, false>, grid, block, 0, stream, p);
  const cudaError_t e = silu ? launch_pdl(conv_forward_kernel<E, W, K, true>, grid, block, 0, stream, p)
                             : launch_pdl(conv_forward_kernel<E, W, K, false>, grid, block, 0, stream, p);
  if (e != cudaSuccess || whole || !state_last) return e;
  p.state_last = state_last;
  return launch_pdl(conv_state_kernel<E, W>, dim3(unsigned((B * p.D + 127) / 128)), dim3(128), 0, stream, p, B * p.D);
}

template <typename E>
cudaError_t launch_conv(const ConvArgs& p, int form, int64_t B, int W, bool fours, bool backward, cudaStream_t stream) {
  if (fours)
    return W == 2   ? launch_conv_as<E, 2, 4>(p, form, B, backward, stream)
           : W == 3 ? launch_conv_as<E, 3, 4>(p, form, B, backward, stream)
                    : launch_conv_as<E, 4, 4>(p, form, B, backward, stream);
  return W == 2   ? launch_conv_as<E, 2, 1>(p, form, B, backward, stream)
         : W == 3 ? launch_conv_as<E, 3, 1>(p, form, B, backward, stream)
                  : launch_conv_as<E, 4, 1>(p, form, B, backward, stream);
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

extern "C" {

int gem_conv_forward(int dtype, int form, int64_t B, int64_t T, int64_t D, int W, const gem_seq_t* x,
                     const float* weight, const float* bias, const float* state,
                     const int32_t* lengths, const uint8_t* reset, const gem_seq_t* y,
                     float* state_last, void* stream) {
  if (!dtype_ok(dtype) || (form != GEM_CONV_LINEAR && form != GEM_CONV_SILU) || !conv_sizes_ok(B, T, D, W)) return GEM_EINVAL;
  if (!input_ok(x, dtype, B, T, D) || !output_ok(y, dtype, B, T, D)) return GEM_EINVAL;
  if (!optional_ok(bias) || !optional_ok(state) || !optional_ok(lengths) || !optional_ok(state_last)) return GEM_EINVAL;
  if (B == 0 || D == 0 || (T == 0 && !state_last)) return GEM_OK;
  if (!array_ok(weight)) return GEM_EINVAL;
  ConvArgs p = {};
  p.x = *x;
  p.y = *y;
  p.weight = weight;
  p.bias = bias;
  p.state = state;
  p.state_last = state_last;
  p.lengths = lengths;
  p.reset = reset;
  p.T = T;
  p.D = int(D);
  const bool fours = in_fours(p.x, dtype, B, T, D) && in_fours(p.y, dtype, B, T, D);
  return launch_status(BY_TYPE(launch_conv, p, form, B, W, fours, false, static_cast<cudaStream_t>(stream)));
}

int64_t gem_conv_workspace(int64_t B, int64_t T, int64_t D, int W) {
  if (!conv_sizes_ok(B, T, D, W)) return -1;
  return B * conv_cut(T).blocks * (W + 1) * D;
}

int gem_conv_backward(int dtype, int form, int64_t B, int64_t T, int64_t D, int W,
                      const gem_seq_t* x, const float* weight, const float* bias,
                      const float* state, const int32_t* lengths, const uint8_t* reset,
                      const gem_seq_t* dy, const float* dstate_last, const gem_seq_t* dx,
                      float* dweight, float* dbias, float* dstate, float* workspace, void* stream) {
  if (!dtype_ok(dtype) || (form != GEM_CONV_LINEAR && form != GEM_CONV_SILU) || !conv_sizes_ok(B, T, D, W)) return GEM_EINVAL;
  if (!input_ok(x, dtype, B, T, D) || !input_ok(dy, dtype, B, T, D) || !output_ok(dx, dtype, B, T, D)) return GEM_EINVAL;
  if (!optional_ok(bias) || !optional_ok(state) || !optional_ok(lengths) || !optional_ok(dstate_last)) return GEM_EINVAL;
  if (!optional_ok(dweight) || !optional_ok(dbias) || !optional_ok(dstate) || !optional_ok(workspace)) return GEM_EINVAL;
  if (dstate && dstate == dstate_last) return GEM_EINVAL;   // (other warps read the one while this one writes the other)
  if (D == 0) return GEM_OK;
  if (B > 0 && !array_ok(weight)) return GEM_EINVAL;
  const bool sums = dweight || dbias;
  if (B > 0 && sums && !workspace) return GEM_EINVAL;
  ConvArgs p = {};
  p.x = *x;
  p.y = *dx;
  p.dy = *dy;
  p.weight = weight;
  p.bias = bias;
  p.state = state;
  p.dstate_last = dstate_last;
  p.dstate = dstate;
  p.partial = sums ? workspace : nullptr;
  p.lengths = lengths;
  p.reset = reset;
  p.T = T;
  p.D = int(D);
  const cudaStream_t on = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (B > 0) {
    const bool fours = in_fours(p.x, dtype, B, T, D) && in_fours(p.dy, dtype, B, T, D) && in_fours(p.y, dtype, B, T, D);
    e = BY_TYPE(launch_conv, p, form, B, W, fours, true, on);
  }
  if (e == cudaSuccess && sums)
    e = launch_pdl(conv_join_kernel, dim3(unsigned((D + 127) / 128), unsigned(W + 1)), dim3(128), 0, on,
                   static_cast<const float*>(workspace), B * conv_cut(T).blocks, int(D), W, dweight, dbias);
  return launch_status(e);
}

}  // extern "C"
