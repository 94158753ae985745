// Selective state space scan: the calls of include/gem_lm.h (argument checks, cuts and dispatch).
#include <algorithm>

#include "lm_ssm.h"

namespace gem {
namespace lm {
namespace ssm {

// Time is split where a block for every sequence and its channels would leave too few warps on an SM.  A split's first pass
// costs 60% of the forward one's second, 20% of the backward one's, so the forward pass is split below one and a half
// blocks an SM, the backward one below two and a half of four; then into whole turns of the blocks that an SM holds, up to three
// while a block has no more than 40 splits to compose, but into no more splits than 128 steps go into, rounded up.  (Rounded down, the backward
// call of 1 x 129 x 512 bf16 takes 33 us instead of 26, of 1 x 200 x 2048 49 instead of 37; the forward ones 10.2, 10.5 and 14.2, 13.8.)  Both calls,
// bf16, 16 states, in us with 1, 4, 8, 16 and 32 splits: 4 x 2048 x 2048 739, 639, 621, 650, 771; 1 x 16,384 x 2048 4711, 1930, 1433,
// 1275, 1258; 8 x 2048 x 2048 1125, 1180, 1178, 1259, 1510.  1 x 50,021 x 512 with 38 (one turn) 955, with 64 1012.
SsmCut ssm_cut(int64_t B, int64_t T, int64_t D, int G, int CH, bool backward, int resident) {
  constexpr int64_t kSms = 152, kMostComposed = 40, kMostSplits = 64, kLeastSteps = 128;
  SsmCut c;
  c.blocks = (D / G + CH - 1) / CH;
  const int64_t base = B * G * c.blocks, turn = resident * kSms;
  const int64_t enough = backward && resident > 2 ? 5 * kSms / 2 : 3 * kSms / 2;
  int64_t splits = 1;
  if (base > 0 && base < enough) {
    int64_t turns = 3;
    while (turns > 1 && turns * turn / base > kMostComposed) --turns;
    splits = std::min(turns * turn / base, kMostSplits);
  }
  splits = std::max(std::min(splits, (T + kLeastSteps - 1) / kLeastSteps), int64_t(1));
  c.steps = ((T + splits - 1) / splits + kTile - 1) / kTile * kTile;
  if (c.steps == 0) c.steps = kTile;
  c.splits = std::max((T + c.steps - 1) / c.steps, int64_t(1));
  return c;
}

namespace {

bool ssm_sizes_ok(int64_t B, int64_t T, int64_t D, int N, int G) {
  if (!extent_ok(B) || !extent_ok(T) || !channels_ok(D) || N < 1 || N > GEM_SSM_STATES || G < 1 || D % G != 0) return false;
  if (!channels_ok(int64_t(G) * N)) return false;
  if (G > D && D > 0) return false;
  if (B == 0 || D == 0) return true;
  // grids: a block at least for 8 channels of a group (and few more where time is split), a thread for each
  // value of db and dc; and the workspace's floats
  if ((D / G / 8 + 1) * G > (kMaxExtent >> 1) / B) return false;
  return T == 0 || (G <= kMaxExtent / B / T && D <= (int64_t(1) << 40) / B / T);
}

bool optional_seq_ok(const gem_seq_t& s, int dtype, int64_t B, int64_t T, int64_t D, bool output) {
  return output ? output_ok(&s, dtype, B, T, D) : input_ok(&s, dtype, B, T, D);
}

bool inputs_ok(int dtype, const gem_ssm_t* in) {
  if (!dtype_ok(dtype) || !in || !ssm_sizes_ok(in->B, in->T, in->D, in->N, in->G)) return false;
  const int64_t states = int64_t(in->G) * in->N;
  if (!input_ok(&in->x, dtype, in->B, in->T, in->D) || !input_ok(&in->dt, dtype, in->B, in->T, in->D)) return false;
  if (in->D > 0 && (!input_ok(&in->b, dtype, in->B, in->T, states) || !input_ok(&in->c, dtype, in->B, in->T, states))) return false;
  if (in->z.data && !input_ok(&in->z, dtype, in->B, in->T, in->D)) return false;
  if (in->B > 0 && in->D > 0 && !array_ok(in->A)) return false;
  return optional_ok(in->skip) && optional_ok(in->dt_bias) && optional_ok(in->lengths);
}

// Whether the pieces of V channels, or states, that blocks read lie at multiples of their size (16 bytes at most).
bool in_pieces(const gem_seq_t& s, int dtype, const gem_ssm_t& in, int V) {
  const int64_t e = dtype_size(dtype), bytes = std::min(int64_t(16), V * e), per = bytes / e;
  return aligned_to(s.data, size_t(bytes)) && (in.B <= 1 || s.stride_b % per == 0) && (in.T <= 1 || s.stride_t % per == 0);
}
bool inputs_wide(const gem_ssm_t& in, int dtype, int V) {
  return in.N % kQuad == 0 && in.D / in.G % V == 0 && in_pieces(in.x, dtype, in, V) && in_pieces(in.dt, dtype, in, V) &&
         (!in.z.data || in_pieces(in.z, dtype, in, V)) && in_pieces(in.b, dtype, in, kQuad) && in_pieces(in.c, dtype, in, kQuad) &&
         aligned_to(in.A, 16);
}

int64_t split_floats(const gem_ssm_t& in, const SsmCut& c) { return c.splits > 1 ? in.B * c.splits * in.D * (int64_t(in.N) + 1) : 0; }

int64_t workspace_floats(const gem_ssm_t& in, bool backward) {
  if (in.B == 0 || in.D == 0) return 0;
  const int64_t forward = split_floats(in, ssm_cut(in.B, in.T, in.D, in.G, block_channels(in.N, kForwardK), false, 4));
  if (!backward) return forward;
  const int LS = state_lanes(in.N);
  const SsmCut c = ssm_cut(in.B, in.T, in.D, in.G, block_channels(in.N, backward_k(LS)), true, backward_resident(LS));
  const int64_t parts = c.blocks > 1 ? in.B * in.T * in.G * c.blocks * 2 * kQuad * state_lanes(in.N) + 3 : 0;   // (and to a multiple of 16 bytes)
  return std::max(forward, split_floats(in, c) + parts + in.B * c.splits * in.D * (int64_t(in.N) + 2));
}

}  // namespace
}  // namespace ssm
}  // namespace lm
}  // namespace gem

using namespace gem::lm;
using namespace gem::lm::ssm;

extern "C" {

int64_t gem_ssm_saved_count(int64_t B, int64_t T, int64_t D, int N) {
  if (!ssm_sizes_ok(B, T, D, N, 1)) return -1;
  return B * ((T + kTile - 1) / kTile) * D * N;
}

int64_t gem_ssm_workspace(int64_t B, int64_t T, int64_t D, int N, int G, int backward) {
  if (!ssm_sizes_ok(B, T, D, N, G)) return -1;
  gem_ssm_t in = {};
  in.B = B;
  in.T = T;
  in.D = D;
  in.N = N;
  in.G = G;
  return workspace_floats(in, backward != 0);
}

int gem_ssm_forward(int dtype, const gem_ssm_t* in, const float* h0, const gem_seq_t* y,
                    float* h_last, float* saved, float* workspace, void* stream) {
  if (!inputs_ok(dtype, in) || !output_ok(y, dtype, in->B, in->T, in->D)) return GEM_EINVAL;
  if (!optional_ok(h0) || !optional_ok(h_last) || !optional_ok(saved) || !optional_ok(workspace)) return GEM_EINVAL;
  if (in->B == 0 || in->D == 0 || (in->T == 0 && !h_last)) return GEM_OK;
  if (workspace_floats(*in, false) > 0 && !workspace) return GEM_EINVAL;
  SsmArgs p = {};
  p.in = *in;
  p.y = *y;
  p.h0 = h0;
  p.h_last = h_last;
  p.saved = saved;
  p.states = workspace;
  const int V = block_channels(in->N, kForwardK) / 8;
  p.wide = inputs_wide(*in, dtype, V) && in_pieces(*y, dtype, *in, V) && aligned_to(h0, 16) && aligned_to(h_last, 16) && aligned_to(saved, 16) &&
           aligned_to(workspace, 16);
  return launch_status(BY_TYPE(launch_forward, p, static_cast<cudaStream_t>(stream)));
}

int gem_ssm_backward(int dtype, const gem_ssm_t* in, const float* saved, const gem_seq_t* dy,
                     const float* dh_last, const gem_ssm_grad_t* out, float* workspace,
                     void* stream) {
  if (!inputs_ok(dtype, in) || !out || !input_ok(dy, dtype, in->B, in->T, in->D)) return GEM_EINVAL;
  const int64_t states = int64_t(in->G) * in->N;
  if (!output_ok(&out->dx, dtype, in->B, in->T, in->D) || !output_ok(&out->ddt, dtype, in->B, in->T, in->D)) return GEM_EINVAL;
  if (in->z.data && !output_ok(&out->dz, dtype, in->B, in->T, in->D)) return GEM_EINVAL;
  if (in->D > 0 && (!output_ok(&out->db, dtype, in->B, in->T, states) || !output_ok(&out->dc, dtype, in->B, in->T, states))) return GEM_EINVAL;
  if (!optional_ok(saved) || !optional_ok(dh_last) || !optional_ok(workspace)) return GEM_EINVAL;
  if (!optional_ok(out->dA) || !optional_ok(out->dskip) || !optional_ok(out->ddt_bias) || !optional_ok(out->dh0)) return GEM_EINVAL;
  const bool params = out->dA || out->dskip || out->ddt_bias;
  if (in->D == 0 || (in->B == 0 && !params)) return GEM_OK;
  if (in->B > 0 && ((in->T > 0 && !saved) || (workspace_floats(*in, true) > 0 && !workspace))) return GEM_EINVAL;
  SsmArgs p = {};
  p.in = *in;
  p.dy = *dy;
  p.dx = out->dx;
  p.ddt = out->ddt;
  p.db = out->db;
  p.dc = out->dc;
  p.dz = out->dz;
  p.h0 = dh_last;
  p.h_last = out->dh0;
  p.saved = const_cast<float*>(saved);
  p.dA = out->dA;
  p.dskip = out->dskip;
  p.ddt_bias = out->ddt_bias;
  p.states = workspace;
  p.params = params;
  const int V = block_channels(in->N, backward_k(state_lanes(in->N))) / 8;
  p.wide = inputs_wide(*in, dtype, V) && in_pieces(*dy, dtype, *in, V) && in_pieces(out->dx, dtype, *in, V) && in_pieces(out->ddt, dtype, *in, V) &&
           (!in->z.data || in_pieces(out->dz, dtype, *in, V)) && aligned_to(dh_last, 16) && aligned_to(out->dh0, 16) && aligned_to(saved, 16) &&
           aligned_to(workspace, 16);
  return launch_status(BY_TYPE(launch_backward, p, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
