// Selective state space scan, backward kernels (internal).
//
// With dy' = dy z sigmoid(z) and g_t the gradient of h_t, from the last step to the first
//
//   g += c_t dy'_t;  dc_t = sum_channels dy'_t h_t;  db_t = sum_channels g step_t x_t
//   q = g exp(step_t A) h_{t-1};  dA += q step_t;  dstep_t = sum_n A q + x_t sum_n g b_t
//   dx_t = step_t sum_n g b_t + skip dy'_t;  g = exp(step_t A) g
//
// A tile is taken in two halves, the later one first: its states are computed again from the one saved before the tile and
// stay in registers (all sixteen would leave fewer warps on an SM).  What a step gives to db and dc goes through shared
// memory, where threads add up the block's channels for a quad of states (exchanges between lanes, two
// selections, a shuffle and a sum for each value, took twice the instructions: 1.07 ms instead of 0.81 with the halves); a
// second kernel adds up the blocks.  The parameters' gradients are summed over a split in registers, then by that kernel
// as well.  Splits are composed from the last one back, as in the forward pass.
//
// Per state and step 28 instructions of a thread, two and a half exponentials among them.  8 x 2048 x 2048 x 16 bf16 with a gate: 0.80
// ms, 0.53 of the issue slots and 59% of shared memory's cycles with 13 warps an SM, whose latencies bound it (HBM 11%).  The registers
// do not quite suffice: 48 bytes a thread are spilled in that kernel, 170 where single elements are loaded (fp32 148, 212), 56 and 80
// with 64 states.
#pragma once

#include "lm_ssm.h"

namespace gem {
namespace lm {
namespace ssm {

__device__ __forceinline__ Vec<2> scaled(const Vec<2>& a, float b) { return a * splat<2>(b); }

constexpr int kHalf = kTile / 2;

// What a step gives to db and dc, [kHalf][lane of channels][2 LS] quads of states, rotated by LS / 4 quads a lane: the eight lanes that
// store together then lie in different banks.
template <typename S>
struct Given {
  static constexpr int kRows = S::CH / S::K, kQuads = 2 * S::LS, kTurn = S::LS / 4, kFloats = kHalf * kRows * kQuads * kQuad;
  static __device__ __forceinline__ int place(int t, int row, int q) {
    return ((t * kRows + row) * kQuads + (q + kTurn * row) % kQuads) * kQuad;
  }
};

template <typename E, int LS, int K, bool WIDE, bool GATE, bool STATES>
__global__ void __launch_bounds__(kSsmThreads, STATES ? 4 : kBackwardResident<LS>) ssm_backward_kernel(const SsmArgs p) {
  using S = Shape<LS, K>;
  constexpr int kSums = GATE ? 3 : 2, U = S::U;
  extern __shared__ float4 shared[];
  float* const given = reinterpret_cast<float*>(shared);
  __shared__ float2 steps[kTile][S::row];                  // (step, step x)
  __shared__ float gys[kTile][S::row];                     // dy'
  __shared__ float4 bc[(STATES ? 1 : 2) * kTile * LS];
  __shared__ float sums[STATES ? 1 : kSums][kTile][S::row];   // sum A2 q, sum g b, sum c h
  pdl_entry();
  const Place<S> a(p);
  if (STATES && a.split == 0) return;
  const int64_t D = p.in.D, N = a.states;
  const int64_t end = min(a.end, a.n), row = a.b * p.splits + a.split;
  // the places of what the thread gives, and from one step to the next
  constexpr int kGivenStep = Given<S>::kRows * Given<S>::kQuads * kQuad;
  const int given_row = threadIdx.x / 32 * S::lanes + threadIdx.x % S::lanes;
  const int to_db = Given<S>::place(0, given_row, a.g), to_dc = Given<S>::place(0, given_row, S::LS + a.g);

  Quad A2[K], g[K], dA[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    A2[k] = a.has(k) ? load_quad<WIDE>(p.in.A + a.state(0, D, k), a.quads) : zeros();
    A2[k] = {scaled(A2[k].a, kLog2e), scaled(A2[k].b, kLog2e)};
    g[k] = dA[k] = zeros();
    if (!a.has(k)) continue;
    if (p.splits == 1 || (STATES && a.split + 1 == p.splits)) {
      if (p.h0) g[k] = load_quad<WIDE>(p.h0 + a.state(a.b, D, k), a.quads);
      // (the second pass's own copy: dh0 may be dh_last)
      if (STATES) store_quad<WIDE>(p.states + a.state(a.b * p.splits, D, k), a.quads, g[k]);
    } else if (!STATES) {
      if (a.split + 1 == p.splits) g[k] = load_quad<WIDE>(p.states + a.state(a.b * p.splits, D, k), a.quads);
#pragma unroll 4
      for (int q = p.splits - 1; q > a.split; --q) {
        const int64_t from = a.b * p.splits + q;
        const Quad first = load_quad<WIDE>(p.states + a.state(from, D, k), a.quads);
        const float sum = p.sums[from * D + a.d0 + a.channel(k)];
        g[k] = sum == INFINITY || q == p.splits - 1 ? first : after_split(sum, A2[k], g[k], first);
      }
    }
  }

  Vec<U> bias[S::V / U], skip[S::V / U], dskip[S::V / U], dbias[S::V / U];
#pragma unroll
  for (int j = 0; j < S::V; ++j) {
    bias[j / U].v[j % U] = p.in.dt_bias && j < a.there ? p.in.dt_bias[a.d0 + a.c0 + j] : 0.0f;
    skip[j / U].v[j % U] = !STATES && p.in.skip && j < a.there ? p.in.skip[a.d0 + a.c0 + j] : 0.0f;
    dskip[j / U].v[j % U] = dbias[j / U].v[j % U] = 0.0f;
  }
  float total[K] = {};
  bool dropped = false;

  Raw<E, S::V, WIDE> x, dt, z, dy, x_next, dt_next, z_next, dy_next;
  States<E, S, WIDE, !STATES, true> b_next;
  Quad start[K], start_next[K];
#pragma unroll
  for (int k = 0; k < K; ++k) start_next[k] = zeros();
  const int64_t chunks = (p.in.T + kTile - 1) / kTile;
  auto load = [&](int64_t t0) {
    const int64_t t = t0 + a.s;
    const int there = t < end ? a.there : 0, d = a.d0 + a.c0;
    if (!STATES) x_next.read(at<E>(p.in.x, a.b, t, d), there);
    dt_next.read(at<E>(p.in.dt, a.b, t, d), there);
    if (GATE) z_next.read(at<E>(p.in.z, a.b, t, d), there);
    dy_next.read(at<E>(p.dy, a.b, t, d), there);
    b_next.load(p, a, t0);
    if (!STATES)
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (a.has(k)) start_next[k] = load_quad<WIDE>(p.saved + a.state(a.b * chunks + t0 / kTile, D, k), a.quads);
  };
  const int64_t tiles = end > a.first ? (end - a.first + kTile - 1) / kTile : 0;
  if (tiles > 0) load(a.first + (tiles - 1) * kTile);
  for (int64_t t0 = a.first + (tiles - 1) * kTile; t0 >= a.first; t0 -= kTile) {
    if (!STATES) x = x_next;
    dt = dt_next;
    if (GATE) z = z_next;
    dy = dy_next;
#pragma unroll
    for (int k = 0; k < K; ++k) start[k] = start_next[k];
    const bool in = t0 + a.s < end;
#pragma unroll
    for (int j = 0; j < S::V; j += U) {
      Vec<U> step = dt.template at<U>(j) + bias[j / U];
      if (p.in.softplus) step = softplus<U>(step);
      if (!in) step = splat<U>(0.0f);
      Vec<U> gy = dy.template at<U>(j);   // (x, z and dy are 0 past the end)
      if (GATE) {
        const Vec<U> zj = z.template at<U>(j);
        gy = gy * (zj * sigmoid<U>(zj));
      }
      Vec<U> input = splat<U>(0.0f);
      if (!STATES) input = step * x.template at<U>(j);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        steps[a.s][(j + i) * 8 + a.o] = {step.v[i], input.v[i]};
        gys[a.s][(j + i) * 8 + a.o] = gy.v[i];
      }
    }
    b_next.stage(bc);
    const unsigned resets = resets_of(p, a.b, t0, end);
    __syncthreads();
    if (t0 > a.first) load(t0 - kTile);
    const int count = int(min(end - t0, int64_t(kTile)));
    dropped |= resets != 0;
    Quad more[K];
#pragma unroll
    for (int k = 0; k < K; ++k) more[k] = nudges(steps[0][a.pos + k * S::lanes].x, A2[k]);

    if constexpr (STATES) {
      auto tile = [&](auto check) {
#pragma unroll
        for (int t = kTile - 1; t >= 0; --t) {
          if (check.value && t >= count) continue;
          const Quad c = quad(bc[t * LS + a.g]);
#pragma unroll
          for (int k = 0; k < K; ++k) {
            const float step = steps[t][a.pos + k * S::lanes].x, gy = gys[t][a.pos + k * S::lanes];
            g[k].a = decay(step, A2[k].a, more[k].a) * fma<2>(c.a, splat<2>(gy), g[k].a);
            g[k].b = decay(step, A2[k].b, more[k].b) * fma<2>(c.b, splat<2>(gy), g[k].b);
            if (check.value && (resets >> t & 1)) g[k] = zeros();
            total[k] += step;
          }
        }
      };
      if (count == kTile && resets == 0)
        tile(std::false_type());
      else
        tile(std::true_type());
      __syncthreads();
    } else {
      // a step forward
      auto forward = [&](int t, Quad (&now)[K], auto check) {
        const Quad b = quad(bc[t * LS + a.g]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const float2 v = steps[t][a.pos + k * S::lanes];
          now[k].a = fma<2>(decay(v.x, A2[k].a, more[k].a), now[k].a, splat<2>(v.y) * b.a);
          now[k].b = fma<2>(decay(v.x, A2[k].b, more[k].b), now[k].b, splat<2>(v.y) * b.b);
          // (not 0 times a decay, which may be infinite)
          if (check.value && (resets >> t & 1)) now[k] = {splat<2>(v.y) * b.a, splat<2>(v.y) * b.b};
        }
      };
      // half: steps from t1 on, whose states are computed again into h from the one before them
      auto half = [&](int t1, const Quad (&before)[K], auto check) {
        Quad h[kHalf][K], now[K];
#pragma unroll
        for (int k = 0; k < K; ++k) now[k] = before[k];
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          if (!check.value || t1 + i < count) forward(t1 + i, now, check);
#pragma unroll
          for (int k = 0; k < K; ++k) h[i][k] = now[k];
        }
        // (the decays are computed again: kept from the first loop they would take the registers of as many states)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            asm volatile("" : "+f"(A2[k].a.v[i]));
            asm volatile("" : "+f"(A2[k].b.v[i]));
          }
        constexpr int kSet = LS < kHalf ? LS : kHalf;   // steps whose sums over the states' lanes are taken together
        float sq[K][kSet], sb[K][kSet], sy[K][kSet];
#pragma unroll
        for (int i = kHalf - 1; i >= 0; --i) {
          const int t = t1 + i;
#pragma unroll
          for (int k = 0; k < K; ++k) sq[k][i % kSet] = sb[k][i % kSet] = sy[k][i % kSet] = 0.0f;
          if (!check.value || t < count) {
            const Quad b = quad(bc[t * LS + a.g]), c = quad(bc[(kTile + t) * LS + a.g]);
            const bool drop = check.value && (resets >> t & 1);
            Quad db = zeros(), dc = zeros();
#pragma unroll
            for (int k = 0; k < K; ++k) {
              const float2 v = steps[t][a.pos + k * S::lanes];
              const float gy = gys[t][a.pos + k * S::lanes];
              const Quad now_h = h[i][k];
              if (GATE) {
                const Vec<2> m = fma<2>(c.b, now_h.b, c.a * now_h.a);
                sy[k][i % kSet] = m.v[0] + m.v[1];
              }
              g[k].a = fma<2>(c.a, splat<2>(gy), g[k].a);
              g[k].b = fma<2>(c.b, splat<2>(gy), g[k].b);
              if (k == 0) {
                db = {scaled(g[k].a, v.y), scaled(g[k].b, v.y)};
                dc = {scaled(now_h.a, gy), scaled(now_h.b, gy)};
              } else {
                db = {fma<2>(g[k].a, splat<2>(v.y), db.a), fma<2>(g[k].b, splat<2>(v.y), db.b)};
                dc = {fma<2>(now_h.a, splat<2>(gy), dc.a), fma<2>(now_h.b, splat<2>(gy), dc.b)};
              }
              const Vec<2> mb = fma<2>(g[k].b, b.b, g[k].a * b.a);
              sb[k][i % kSet] = mb.v[0] + mb.v[1];
              Quad prev = before[k];
              if (i > 0) prev = h[i > 0 ? i - 1 : 0][k];
              if (drop) prev = zeros();
              g[k].a = g[k].a * decay(v.x, A2[k].a, more[k].a);
              g[k].b = g[k].b * decay(v.x, A2[k].b, more[k].b);
              const Vec<2> q0 = g[k].a * prev.a, q1 = g[k].b * prev.b;
              const Vec<2> mq = fma<2>(q1, A2[k].b, q0 * A2[k].a);
              sq[k][i % kSet] = drop ? 0.0f : mq.v[0] + mq.v[1];
              if (drop) {
                g[k] = zeros();
              } else {
                dA[k].a = fma<2>(q0, splat<2>(v.x), dA[k].a);
                dA[k].b = fma<2>(q1, splat<2>(v.x), dA[k].b);
              }
            }
            *reinterpret_cast<float4*>(given + to_db + i * kGivenStep) = make_float4(db.a.v[0], db.a.v[1], db.b.v[0], db.b.v[1]);
            *reinterpret_cast<float4*>(given + to_dc + i * kGivenStep) = make_float4(dc.a.v[0], dc.a.v[1], dc.b.v[0], dc.b.v[1]);
          }
          if (i % kSet == 0) {
            // (with more lanes than steps of a half, the lanes that end up with the same step write the same)
            const int s = t + a.g * kSet / LS;
#pragma unroll
            for (int k = 0; k < K; ++k) {
              scatter_sums<kSet, 16, S::lanes>(sq[k]);
              scatter_sums<kSet, 16, S::lanes>(sb[k]);
              if (GATE) scatter_sums<kSet, 16, S::lanes>(sy[k]);
              sums[0][s][a.pos + k * S::lanes] = sq[k][0];
              sums[1][s][a.pos + k * S::lanes] = sb[k][0];
              if (GATE) sums[kSums - 1][s][a.pos + k * S::lanes] = sy[k][0];
            }
          }
        }
      };
      // the half's db and dc of all the block's channels: a thread for a quad of states of a step, or kShare of them
      // with a share of the channels each, which begin a rotation apart
      auto collect = [&](int t1) {
        constexpr int kQuads = Given<S>::kQuads, kShare = LS < 8 ? 8 / LS : 1, kEach = Given<S>::kRows / kShare;
#pragma unroll
        for (int i = 0; i < kHalf * kQuads * kShare / kSsmThreads; ++i) {
          const int o = (i * kSsmThreads + threadIdx.x) / kShare, share = threadIdx.x % kShare, t = o / kQuads, q = o % kQuads;
          Quad v = zeros();
#pragma unroll
          for (int c = 0; c < kEach; ++c) {
            const int channel = share * kEach + (c + share * (kQuads / kShare)) % kEach;
            const Quad w = quad(*reinterpret_cast<const float4*>(given + Given<S>::place(t, channel, q)));
            v = {v.a + w.a, v.b + w.b};
          }
#pragma unroll
          for (int bit = 1; bit < kShare; bit *= 2)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              v.a.v[k] += __shfl_xor_sync(~0u, v.a.v[k], bit);
              v.b.v[k] += __shfl_xor_sync(~0u, v.b.v[k], bit);
            }
          if (share != 0 || t1 + t >= count) continue;
          const int64_t step = t0 + t1 + t;
          if (p.blocks > 1) {
            store_quad<true>(p.bc_part + ((((a.b * p.in.T + step) * p.in.G + a.group) * p.blocks + a.part) * kQuads + q) * kQuad, kQuad, v);
          } else {
            E* const to = at<E>(q < LS ? p.db : p.dc, a.b, step, a.group * a.states + q % LS * kQuad);
            const int there = a.states - q % LS * kQuad;
            const float out[kQuad] = {v.a.v[0], v.a.v[1], v.b.v[0], v.b.v[1]};
#pragma unroll
            for (int k = 0; k < kQuad; ++k)
              if (k < there) to[k] = from_f32<E>(out[k]);
          }
        }
      };
      auto tile = [&](auto check) {
        if (!check.value || count > kHalf) {
          Quad middle[K];
#pragma unroll
          for (int k = 0; k < K; ++k) middle[k] = start[k];
#pragma unroll
          for (int t = 0; t < kHalf; ++t) forward(t, middle, check);
          half(kHalf, middle, check);
          __syncthreads();
          collect(kHalf);
          __syncthreads();
        }
        half(0, start, check);
      };
      if (count == kTile && resets == 0)
        tile(std::false_type());
      else
        tile(std::true_type());
      __syncthreads();
      collect(0);

      if (t0 + a.s < a.end) {
        float out[3][S::V];
#pragma unroll
        for (int j = 0; j < S::V; j += U) {
          Vec<U> sq, sb, sy, gy, step;
#pragma unroll
          for (int k = 0; k < U; ++k) {
            const int i = (j + k) * 8 + a.o;
            sq.v[k] = sums[0][a.s][i];
            sb.v[k] = sums[1][a.s][i];
            sy.v[k] = sums[kSums - 1][a.s][i];
            gy.v[k] = gys[a.s][i];
            step.v[k] = steps[a.s][i].x;
          }
          const Vec<U> xj = x.template at<U>(j);
          Vec<U> d = fma<U>(sb, xj, sq * splat<U>(kLn2));
          if (p.in.softplus) d = d * sigmoid<U>(dt.template at<U>(j) + bias[j / U]);
          const Vec<U> dx = fma<U>(sb, step, skip[j / U] * gy);
          Vec<U> dz = d;
          if (GATE) {
            const Vec<U> zj = z.template at<U>(j), s = sigmoid<U>(zj), one = splat<U>(1.0f);
            dz = dy.template at<U>(j) * fma<U>(skip[j / U], xj, sy) * (s * fma<U>(zj, one - s, one));
          }
          if (in) {
            dskip[j / U] = fma<U>(gy, xj, dskip[j / U]);
            dbias[j / U] = dbias[j / U] + d;
          }
#pragma unroll
          for (int k = 0; k < U; ++k) {
            out[0][j + k] = in ? dx.v[k] : 0.0f;
            out[1][j + k] = in ? d.v[k] : 0.0f;
            out[2][j + k] = in ? dz.v[k] : 0.0f;
          }
        }
        const int64_t t = t0 + a.s;
        const int d = a.d0 + a.c0;
        store_piece<E, S::V, WIDE>(at<E>(p.dx, a.b, t, d), a.there, out[0]);
        store_piece<E, S::V, WIDE>(at<E>(p.ddt, a.b, t, d), a.there, out[1]);
        if (GATE) store_piece<E, S::V, WIDE>(at<E>(p.dz, a.b, t, d), a.there, out[2]);
      }
      __syncthreads();   // (the next tile's steps replace these)
    }
  }
  if constexpr (STATES) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (a.has(k)) {
        store_quad<WIDE>(p.states + a.state(row, D, k), a.quads, g[k]);
        if (a.g == 0) p.sums[row * D + a.d0 + a.channel(k)] = dropped ? INFINITY : total[k];
      }
    return;
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!a.has(k)) continue;
      if (a.split == 0 && p.h_last) store_quad<WIDE>(p.h_last + a.state(a.b, D, k), a.quads, g[k]);
      const float v[kQuad] = {dA[k].a.v[0], dA[k].a.v[1], dA[k].b.v[0], dA[k].b.v[1]};
#pragma unroll
      for (int i = 0; i < kQuad; ++i)
        if (p.params && i < a.quads) p.param_part[(row * (N + 2) + a.g * kQuad + i) * D + a.d0 + a.channel(k)] = v[i];
    }
    if (p.params) {
#pragma unroll
      for (int j = 0; j < S::V; ++j) {
        sums[0][a.s][j * 8 + a.o] = dskip[j / U].v[j % U];
        sums[1][a.s][j * 8 + a.o] = dbias[j / U].v[j % U];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < 2 * S::CH; i += kSsmThreads) {
        const int which = i / S::CH, col = i % S::CH, c = col % 8 * S::V + col / 8;
        float v = 0.0f;
#pragma unroll
        for (int s = 0; s < kTile; ++s) v += sums[which][s][col];
        if (c < a.channels) p.param_part[(row * (N + 2) + N + which) * D + a.d0 + c] = v;
      }
    }
    // what is left of the split past the sequence's end
    const int64_t past = a.first + tiles * kTile;
    const float none[S::V] = {};
    for (int64_t t = past + a.s; t < a.end; t += kTile) {
      const int d = a.d0 + a.c0;
      store_piece<E, S::V, WIDE>(at<E>(p.dx, a.b, t, d), a.there, none);
      store_piece<E, S::V, WIDE>(at<E>(p.ddt, a.b, t, d), a.there, none);
      if (GATE) store_piece<E, S::V, WIDE>(at<E>(p.dz, a.b, t, d), a.there, none);
    }
    if (p.blocks == 1) {
      const int64_t left = a.end - max(end, a.first);
      for (int64_t i = threadIdx.x; i < left * N; i += kSsmThreads) {
        const int64_t t = max(end, a.first) + i / N;
        const int n = a.group * a.states + int(i % N);
        *at<E>(p.db, a.b, t, n) = from_f32<E>(0.0f);
        *at<E>(p.dc, a.b, t, n) = from_f32<E>(0.0f);
      }
    }
  }
}

// db and dc from the blocks' parts, a thread for each value.
template <typename E>
__global__ void __launch_bounds__(256) ssm_join_states_kernel(const SsmArgs p, int NP, int64_t count) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= count) return;
  const int k = int(i % (2 * NP)), n = k % NP;
  if (n >= p.in.N) return;
  const int64_t row = i / (2 * NP);
  const int group = int(row % p.in.G);
  const int64_t t = row / p.in.G % p.in.T, b = row / p.in.G / p.in.T;
  float v = 0.0f;
  if (!p.in.lengths || t < p.in.lengths[b])
#pragma unroll 8
    for (int j = 0; j < p.blocks; ++j) v += p.bc_part[(row * p.blocks + j) * (2 * NP) + k];
  *at<E>(k < NP ? p.db : p.dc, b, t, group * p.in.N + n) = from_f32<E>(v);
}

// dA, dskip and ddt_bias from the splits' parts: 32 channels by a block, of whose WARPS each takes every WARPS-th row.
template <int WARPS>
__global__ void __launch_bounds__(WARPS * 32) ssm_join_params_kernel(const SsmArgs p) {
  __shared__ float sums[WARPS][32];
  pdl_entry();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n = blockIdx.y, N = p.in.N;
  const int64_t d = int64_t(blockIdx.x) * 32 + lane, rows = p.in.B * p.splits;
  float v = 0.0f;
  if (d < p.in.D)
#pragma unroll 8
    for (int64_t r = warp; r < rows; r += WARPS) v += p.param_part[(r * (N + 2) + n) * p.in.D + d];
  sums[warp][lane] = v;
  __syncthreads();
  if (warp != 0 || d >= p.in.D) return;
#pragma unroll
  for (int w = 1; w < WARPS; ++w) v += sums[w][lane];
  if (n < N) {
    if (p.dA) p.dA[d * N + n] = v;
  } else if (n == N) {
    if (p.dskip) p.dskip[d] = v;
  } else if (p.ddt_bias) {
    p.ddt_bias[d] = v;
  }
}

template <typename E, int LS, bool WIDE>
cudaError_t launch_backward_as(SsmArgs p, cudaStream_t stream) {
  using S = Shape<LS, kBackwardK<LS>>;
  const SsmCut cut = ssm_cut(p.in.B, p.in.T, p.in.D, p.in.G, S::CH, true, kBackwardResident<LS>);
  p.blocks = int(cut.blocks);
  p.splits = int(cut.splits);
  p.steps = cut.steps;
  float* space = p.states;
  if (cut.splits > 1) {
    p.sums = space + p.in.B * cut.splits * p.in.D * p.in.N;
    space = p.sums + p.in.B * cut.splits * p.in.D;
  }
  if (cut.blocks > 1) {
    p.bc_part = space + (16 - reinterpret_cast<uintptr_t>(space) % 16) % 16 / 4;   // (quads are stored to it)
    space += p.in.B * p.in.T * p.in.G * cut.blocks * 2 * S::NP + 3;
  }
  p.param_part = space;
  const dim3 grid(unsigned(p.in.B * cut.splits * p.in.G * cut.blocks)), block(kSsmThreads);
  const bool gate = p.in.z.data;
  cudaError_t e = cudaSuccess;
  if (grid.x > 0) {
    constexpr size_t kShared = size_t(Given<S>::kFloats) * 4;
    e = gate ? allow_shared<ssm_backward_kernel<E, LS, kBackwardK<LS>, WIDE, true, false>, false, kShared>(kShared)
             : allow_shared<ssm_backward_kernel<E, LS, kBackwardK<LS>, WIDE, false, false>, false, kShared>(kShared);
    if (e == cudaSuccess && cut.splits > 1)
      e = gate ? launch_pdl(ssm_backward_kernel<E, LS, kBackwardK<LS>, WIDE, true, true>, grid, block, 0, stream, p)
               : launch_pdl(ssm_backward_kernel<E, LS, kBackwardK<LS>, WIDE, false, true>, grid, block, 0, stream, p);
    if (e == cudaSuccess)
      e = gate ? launch_pdl(ssm_backward_kernel<E, LS, kBackwardK<LS>, WIDE, true, false>, grid, block, kShared, stream, p)
               : launch_pdl(ssm_backward_kernel<E, LS, kBackwardK<LS>, WIDE, false, false>, grid, block, kShared, stream, p);
  }
  if (e == cudaSuccess && cut.blocks > 1) {
    const int64_t count = p.in.B * p.in.T * p.in.G * 2 * S::NP;
    if (count > 0) e = launch_pdl(ssm_join_states_kernel<E>, dim3(unsigned((count + 255) / 256)), dim3(256), 0, stream, p, int(S::NP), count);
  }
  if (e == cudaSuccess && p.params) {
    // (us of the whole call, bf16, with 32 warps and with a thread for each value: 4096 x 16 x 256 x 16 462, 1011; 2000 x 33 x 64 x 64 560,
    // 828; 64 x 1024 x 512 x 16 765, 771)
    const dim3 joins(unsigned((p.in.D + 31) / 32), unsigned(p.in.N + 2));
    e = p.in.B * cut.splits > 16 ? launch_pdl(ssm_join_params_kernel<32>, joins, dim3(32 * 32), 0, stream, p)
                                 : launch_pdl(ssm_join_params_kernel<4>, joins, dim3(4 * 32), 0, stream, p);
  }
  return e;
}

template <typename E>
cudaError_t launch_backward(SsmArgs p, cudaStream_t stream) {
  switch (state_lanes(p.in.N)) {
    case 4: return p.wide ? launch_backward_as<E, 4, true>(p, stream) : launch_backward_as<E, 4, false>(p, stream);
    case 8: return p.wide ? launch_backward_as<E, 8, true>(p, stream) : launch_backward_as<E, 8, false>(p, stream);
    default: return p.wide ? launch_backward_as<E, 16, true>(p, stream) : launch_backward_as<E, 16, false>(p, stream);
  }
}

}  // namespace ssm
}  // namespace lm
}  // namespace gem
