// Selective state space scan, forward kernels (internal).
#pragma once

#include "lm_ssm.h"

namespace gem {
namespace lm {
namespace ssm {

// Goes over a split.  STATES: the first pass of a split time, for the last state and the sum of steps alone.  Per state and step 10
// instructions of a thread, an exponential among them (a third of them the staging, whose share falls with N).  8 x 2048 x 2048 x 16 bf16
// with a gate, states saved: 255 us, 0.60 of the issue slots with 13 warps an SM (HBM 18%).
template <typename E, int LS, int K, bool WIDE, bool STATES>
__global__ void __launch_bounds__(kSsmThreads, 4) ssm_forward_kernel(const SsmArgs p) {
  using S = Shape<LS, K>;
  __shared__ float2 steps[kTile][S::row];                          // (step, step x) of each channel
  __shared__ float4 bc[(STATES ? 1 : 2) * kTile * LS];
  __shared__ float mixed[STATES ? 1 : kTile][STATES ? 1 : S::row];   // sum c h
  pdl_entry();
  const Place<S> a(p);
  if (STATES && a.split + 1 == p.splits) return;
  const int64_t D = p.in.D;
  const bool gate = p.in.z.data;
  const int64_t end = min(a.end, a.n), row = a.b * p.splits + a.split;

  Quad A2[K], h[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    A2[k] = a.has(k) ? load_quad<WIDE>(p.in.A + a.state(0, D, k), a.quads) : zeros();
    A2[k] = {A2[k].a * splat<2>(kLog2e), A2[k].b * splat<2>(kLog2e)};
    h[k] = zeros();
  }
  auto state0 = [&](int k) { return p.h0 ? load_quad<WIDE>(p.h0 + a.state(a.b, D, k), a.quads) : zeros(); };
  if (STATES) {
    if (a.split == 0) {
      // (the second pass's own copy: h_last may be h0)
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (a.has(k)) {
          h[k] = state0(k);
          store_quad<WIDE>(p.states + a.state(a.b * p.splits + p.splits - 1, D, k), a.quads, h[k]);
        }
    }
  } else if (p.splits == 1) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (a.has(k)) h[k] = state0(k);
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!a.has(k)) continue;
      if (a.split == 0) h[k] = load_quad<WIDE>(p.states + a.state(a.b * p.splits + p.splits - 1, D, k), a.quads);
#pragma unroll 4
      for (int q = 0; q < a.split; ++q) {
        const int64_t from = a.b * p.splits + q;
        const Quad last = load_quad<WIDE>(p.states + a.state(from, D, k), a.quads);
        const float sum = p.sums[from * D + a.d0 + a.channel(k)];
        h[k] = sum == INFINITY || q == 0 ? last : after_split(sum, A2[k], h[k], last);
      }
    }
  }

  constexpr int U = S::U;
  Vec<U> bias[S::V / U], skip[S::V / U];
#pragma unroll
  for (int j = 0; j < S::V; ++j) {
    bias[j / U].v[j % U] = p.in.dt_bias && j < a.there ? p.in.dt_bias[a.d0 + a.c0 + j] : 0.0f;
    skip[j / U].v[j % U] = !STATES && p.in.skip && j < a.there ? p.in.skip[a.d0 + a.c0 + j] : 0.0f;
  }
  float sum[K] = {};
  bool dropped = false;

  Raw<E, S::V, WIDE> x, dt, z, x_next, dt_next, z_next;
  States<E, S, WIDE, true, !STATES> b_next;
  auto load = [&](int64_t t0) {
    const int64_t t = t0 + a.s;
    const int there = t < end ? a.there : 0, d = a.d0 + a.c0;
    x_next.read(at<E>(p.in.x, a.b, t, d), there);
    dt_next.read(at<E>(p.in.dt, a.b, t, d), there);
    if (!STATES && gate) z_next.read(at<E>(p.in.z, a.b, t, d), there);
    b_next.load(p, a, t0);
  };
  if (a.first < end) load(a.first);
  for (int64_t t0 = a.first; t0 < end; t0 += kTile) {
    x = x_next;
    dt = dt_next;
    z = z_next;
    const bool in = t0 + a.s < end;
#pragma unroll
    for (int j = 0; j < S::V; j += U) {
      Vec<U> step = dt.template at<U>(j) + bias[j / U];
      if (p.in.softplus) step = softplus<U>(step);
      if (!in) step = splat<U>(0.0f);
      const Vec<U> input = step * x.template at<U>(j);   // (x is 0 past the end)
#pragma unroll
      for (int i = 0; i < U; ++i) steps[a.s][(j + i) * 8 + a.o] = {step.v[i], input.v[i]};
    }
    b_next.stage(bc);
    const unsigned resets = resets_of(p, a.b, t0, end);
    __syncthreads();
    if (t0 + kTile < end) load(t0 + kTile);
    if (!STATES && p.saved) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (a.has(k)) store_quad<WIDE>(p.saved + a.state(a.b * ((p.in.T + kTile - 1) / kTile) + t0 / kTile, D, k), a.quads, h[k]);
    }
    float y[K][kTile];
    Quad more[K];
#pragma unroll
    for (int k = 0; k < K; ++k) more[k] = nudges(steps[0][a.pos + k * S::lanes].x, A2[k]);
    auto tile = [&](auto check) {
      const int count = int(min(end - t0, int64_t(kTile)));
      // steps in sets: what a set reads and its decays come first, so that their latencies overlap
      constexpr int kSet = 4;
#pragma unroll
      for (int t1 = 0; t1 < kTile; t1 += kSet) {
        Quad b[kSet], c[kSet];
        float2 v[kSet][K];
#pragma unroll
        for (int i = 0; i < kSet; ++i) {
          b[i] = quad(bc[(t1 + i) * LS + a.g]);
          if (!STATES) c[i] = quad(bc[(kTile + t1 + i) * LS + a.g]);
#pragma unroll
          for (int k = 0; k < K; ++k) v[i][k] = steps[t1 + i][a.pos + k * S::lanes];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
          Quad dec[kSet];
#pragma unroll
          for (int i = 0; i < kSet; ++i) dec[i] = {decay(v[i][k].x, A2[k].a, more[k].a), decay(v[i][k].x, A2[k].b, more[k].b)};
#pragma unroll
          for (int i = 0; i < kSet; ++i) {
            const int t = t1 + i;
            if (!STATES) y[k][t] = 0.0f;
            if (check.value && t >= count) continue;
            h[k].a = fma<2>(dec[i].a, h[k].a, splat<2>(v[i][k].y) * b[i].a);
            h[k].b = fma<2>(dec[i].b, h[k].b, splat<2>(v[i][k].y) * b[i].b);
            // (not 0 times a decay, which may be infinite)
            if (check.value && (resets >> t & 1)) h[k] = {splat<2>(v[i][k].y) * b[i].a, splat<2>(v[i][k].y) * b[i].b};
            if (STATES) {
              sum[k] += v[i][k].x;
            } else {
              const Vec<2> m = fma<2>(c[i].b, h[k].b, c[i].a * h[k].a);
              y[k][t] = m.v[0] + m.v[1];
            }
          }
        }
      }
    };
    if (t0 + kTile <= end && resets == 0)
      tile(std::false_type());
    else
      tile(std::true_type());
    dropped |= resets != 0;
    if (!STATES) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        scatter_sums<kTile, 16, S::lanes>(y[k]);
#pragma unroll
        for (int i = 0; i < kTile / LS; ++i) mixed[a.g * (kTile / LS) + i][a.pos + k * S::lanes] = y[k][i];
      }
    }
    __syncthreads();
    if (!STATES && t0 + a.s < a.end) {
      float out[S::V];
#pragma unroll
      for (int j = 0; j < S::V; j += U) {
        Vec<U> v;
#pragma unroll
        for (int i = 0; i < U; ++i) v.v[i] = mixed[a.s][(j + i) * 8 + a.o];
        v = fma<U>(skip[j / U], x.template at<U>(j), v);
        if (gate) {
          const Vec<U> zj = z.template at<U>(j);
          v = v * (zj * sigmoid<U>(zj));
        }
#pragma unroll
        for (int i = 0; i < U; ++i) out[j + i] = in ? v.v[i] : 0.0f;
      }
      store_piece<E, S::V, WIDE>(at<E>(p.y, a.b, t0 + a.s, a.d0 + a.c0), a.there, out);
    }
  }
  if (STATES) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (a.has(k)) {
        store_quad<WIDE>(p.states + a.state(row, D, k), a.quads, h[k]);
        if (a.g == 0) p.sums[row * D + a.d0 + a.channel(k)] = dropped ? INFINITY : sum[k];
      }
    return;
  }
  if (p.h_last && a.split + 1 == p.splits) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (a.has(k)) store_quad<WIDE>(p.h_last + a.state(a.b, D, k), a.quads, h[k]);
  }
  // what is left of the split past the sequence's end
  const int64_t past = a.first < end ? a.first + (end - a.first + kTile - 1) / kTile * kTile : a.first;
  const float none[S::V] = {};
  for (int64_t t = past + a.s; t < a.end; t += kTile)
    store_piece<E, S::V, WIDE>(at<E>(p.y, a.b, t, a.d0 + a.c0), a.there, none);
}

// One step: a thread for four states of a channel, the LS lanes of a channel side by side, so that states are read and written
// in the order of memory.  (16 x 2048 x 16 bf16: 3.4 us; the kernel above, most of whose tile would be empty, 8.1.)
template <typename E, int LS, bool WIDE>
__global__ void __launch_bounds__(kSsmThreads) ssm_step_kernel(const SsmArgs p) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * kSsmThreads + threadIdx.x, D = p.in.D, N = p.in.N;
  const int q = threadIdx.x % LS;
  const int64_t row = i / LS;
  const bool on = row < p.in.B * D;
  const int64_t b = on ? row / D : 0, d = on ? row % D : 0;
  const int there = on ? min(max(int(N) - q * kQuad, 0), kQuad) : 0;
  const int64_t state = (b * D + d) * N + q * kQuad;
  const int first = int(d / (D / p.in.G) * N) + q * kQuad;
  const bool live = !p.in.lengths || p.in.lengths[b] > 0, gate = p.in.z.data;
  Quad h = zeros();
  if (p.h0) h = load_quad<WIDE>(p.h0 + state, there);
  if (p.saved && live) store_quad<WIDE>(p.saved + state, there, h);
  Raw<E, kQuad, WIDE> bs, cs;
  bs.read(at<E>(p.in.b, b, 0, first), live ? there : 0);
  cs.read(at<E>(p.in.c, b, 0, first), live ? there : 0);
  Quad A2 = load_quad<WIDE>(p.in.A + d * N + q * kQuad, there);
  float x = 0.0f, dt = 0.0f, z = 0.0f;
  if (live) {
    x = to_f32(*at<E>(p.in.x, b, 0, int(d)));
    dt = to_f32(*at<E>(p.in.dt, b, 0, int(d)));
    if (gate) z = to_f32(*at<E>(p.in.z, b, 0, int(d)));
  }
  const float skip = p.in.skip ? p.in.skip[d] : 0.0f;
  float step = dt + (p.in.dt_bias ? p.in.dt_bias[d] : 0.0f);
  if (p.in.softplus) step = softplus<1>({step}).v[0];
  float y = 0.0f;
  if (live) {
    const bool drop = p.in.reset && p.in.reset[b];
    A2 = {A2.a * splat<2>(kLog2e), A2.b * splat<2>(kLog2e)};
    const Vec<2> in = splat<2>(step * x);
    const Quad more = nudges(step, A2);
    const Quad input = {in * bs.template at<2>(0), in * bs.template at<2>(2)};
    h = {fma<2>(decay(step, A2.a, more.a), h.a, input.a), fma<2>(decay(step, A2.b, more.b), h.b, input.b)};
    if (drop) h = input;   // (not 0 times a decay, which may be infinite)
    const Vec<2> m = fma<2>(cs.template at<2>(2), h.b, cs.template at<2>(0) * h.a);
    y = m.v[0] + m.v[1];
  }
  if (p.h_last) store_quad<WIDE>(p.h_last + state, there, h);
#pragma unroll
  for (int bit = LS / 2; bit > 0; bit /= 2) y += __shfl_xor_sync(~0u, y, bit);
  if (!on || q != 0) return;
  y = fmaf(skip, x, y);
  if (gate) y *= z * sigmoid<1>({z}).v[0];
  *at<E>(p.y, b, 0, int(d)) = from_f32<E>(live ? y : 0.0f);
}

template <typename E, int LS, bool WIDE>
cudaError_t launch_forward_as(SsmArgs p, cudaStream_t stream) {
  if (p.in.T == 1)
    return launch_pdl(ssm_step_kernel<E, LS, WIDE>, dim3(unsigned((p.in.B * p.in.D * LS + kSsmThreads - 1) / kSsmThreads)), dim3(kSsmThreads), 0,
                      stream, p);
  using S = Shape<LS, kForwardK>;
  const SsmCut cut = ssm_cut(p.in.B, p.in.T, p.in.D, p.in.G, S::CH, false, 4);
  p.blocks = int(cut.blocks);
  p.splits = int(cut.splits);
  p.steps = cut.steps;
  p.sums = p.states + p.in.B * cut.splits * p.in.D * p.in.N;
  const dim3 grid(unsigned(p.in.B * cut.splits * p.in.G * cut.blocks));
  if (cut.splits > 1) {
    const cudaError_t e = launch_pdl(ssm_forward_kernel<E, LS, kForwardK, WIDE, true>, grid, dim3(kSsmThreads), 0, stream, p);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(ssm_forward_kernel<E, LS, kForwardK, WIDE, false>, grid, dim3(kSsmThreads), 0, stream, p);
}

template <typename E>
cudaError_t launch_forward(SsmArgs p, cudaStream_t stream) {
  switch (state_lanes(p.in.N)) {
    case 4: return p.wide ? launch_forward_as<E, 4, true>(p, stream) : launch_forward_as<E, 4, false>(p, stream);
    case 8: return p.wide ? launch_forward_as<E, 8, true>(p, stream) : launch_forward_as<E, 8, false>(p, stream);
    default: return p.wide ? launch_forward_as<E, 16, true>(p, stream) : launch_forward_as<E, 16, false>(p, stream);
  }
}

}  // namespace ssm
}  // namespace lm
}  // namespace gem
