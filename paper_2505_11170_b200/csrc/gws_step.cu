// Host side of the layer norm and of the AdamW step declared in gws.h: argument validation, choice of kernel and launch geometry; no device
// memory is allocated here.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "gws.h"
#include "gws_adamw.cuh"
#include "gws_host.h"
#include "gws_norm.cuh"

namespace {

// ---- layer norm ------------------------------------------------------------------------------------------------------
int check_norm(const gws_norm_desc* d) {
  if (d == nullptr) return GWS_ERR_NULL;
  const int st = check_dims(d->rows, d->cols, 0);
  if (st != GWS_OK) return st;
  if (d->weight_type != GWS_TYPE_BF16 && d->weight_type != GWS_TYPE_F32) return GWS_ERR_UNSUPPORTED;
  for (const int64_t ld : {d->ld_x, d->ld_residual, d->ld_grad_y, d->ld_grad_sum}) {
    if (ld < 0) return GWS_ERR_SHAPE;
    if (ld > kMaxDim) return GWS_ERR_LIMIT;
  }
  return GWS_OK;
}
int64_t weight_bytes(const gws_norm_desc& d) { return d.weight_type == GWS_TYPE_F32 ? 4 : 2; }

// Whether rows of a BF16 matrix (absent: null) start on 16-byte boundaries.
bool wide_rows(const void* p, int64_t rows, int64_t ld) { return p == nullptr || (on(p, 16) && (rows <= 1 || ld % 8 == 0)); }

// Threads of a row; a block of 256 or more holds one row or several.  0: rows that no block holds.
int norm_team(int64_t cols) {
  for (const int team : {32, 64, 96, 128, 192, 256, 384, 512})
    if (cols <= 16 * team) return team;
  return 0;
}
int64_t norm_teams(int team) { return team < 256 ? 256 / team : 1; }

template <bool WIDE>
int launch_norm_fwd(const NormArgs& a, cudaStream_t s) {
  const char* what = "layer norm kernel";
  const int team = norm_team(a.cols);
  if (team == 0 && a.cols <= 16384) return launch(k_norm_fwd<1024, 2, WIDE>, static_cast<unsigned>(std::min<int64_t>(a.rows, sm_count())), 1024, 0, 1, s, what, a);
  if (team == 0) return launch(k_norm_fwd_long, static_cast<unsigned>(a.rows), kNormLong, 0, 1, s, what, a);
  const int64_t teams = norm_teams(team), fit = static_cast<int64_t>(sm_count()) * norm_blocks(team, WIDE);
  const unsigned grid = static_cast<unsigned>(std::min((a.rows + teams - 1) / teams, fit));
  if (team == 32 && a.cols <= 256) return launch(k_norm_fwd<32, 1, WIDE>, grid, 256, 0, 1, s, what, a);
  if (team == 32) return launch(k_norm_fwd<32, 2, WIDE>, grid, 256, 0, 1, s, what, a);
  if (team == 64) return launch(k_norm_fwd<64, 2, WIDE>, grid, 256, 0, 1, s, what, a);
  if (team == 96) return launch(k_norm_fwd<96, 2, WIDE>, grid, kNormThreads<96>, 0, 1, s, what, a);
  if (team == 128) return launch(k_norm_fwd<128, 2, WIDE>, grid, 256, 0, 1, s, what, a);
  if (team == 192) return launch(k_norm_fwd<192, 2, WIDE>, grid, kNormThreads<192>, 0, 1, s, what, a);
  if (team == 256) return launch(k_norm_fwd<256, 2, WIDE>, grid, 256, 0, 1, s, what, a);
  if (team == 384) return launch(k_norm_fwd<384, 2, WIDE>, grid, 384, 0, 1, s, what, a);
  return launch(k_norm_fwd<512, 2, WIDE>, grid, 512, 0, 1, s, what, a);
}

struct NormBack {
  int team;                      // threads of a row, 0: rows that no block holds
  uint32_t blocks;               // and parts of the column sums
};
NormBack norm_back(int64_t rows, int64_t cols) {
  const int sms = sm_count();
  if (norm_team(cols) == 0) return {0, static_cast<uint32_t>(std::min<int64_t>(64, (rows + 31) / 32))};
  const int team = norm_team(cols);
  const int64_t teams = team < 128 ? 256 / team : std::max(1, 512 / team);
  return {team, static_cast<uint32_t>(std::min<int64_t>((rows + teams - 1) / teams, static_cast<int64_t>(sms) * (team < 128 ? 2 : 1)))};
}
template <bool WIDE>
int launch_norm_bwd(const NormArgs& a, const NormBack& b, cudaStream_t s) {
  const char* what = "layer norm backward kernel";
  if (b.team == 32 && a.cols <= 256) return launch(k_norm_bwd<32, 1, WIDE>, b.blocks, kNormBackThreads<32>, 0, 1, s, what, a);
  if (b.team == 32) return launch(k_norm_bwd<32, 2, WIDE>, b.blocks, kNormBackThreads<32>, 0, 1, s, what, a);
  if (b.team == 64) return launch(k_norm_bwd<64, 2, WIDE>, b.blocks, kNormBackThreads<64>, 0, 1, s, what, a);
  if (b.team == 96) return launch(k_norm_bwd<96, 2, WIDE>, b.blocks, kNormBackThreads<96>, 0, 1, s, what, a);
  if (b.team == 128) return launch(k_norm_bwd<128, 2, WIDE>, b.blocks, kNormBackThreads<128>, 0, 1, s, what, a);
  if (b.team == 192) return launch(k_norm_bwd<192, 2, WIDE>, b.blocks, kNormBackThreads<192>, 0, 1, s, what, a);
  if (b.team == 256) return launch(k_norm_bwd<256, 2, WIDE>, b.blocks, kNormBackThreads<256>, 0, 1, s, what, a);
  if (b.team == 384) return launch(k_norm_bwd<384, 2, WIDE>, b.blocks, kNormBackThreads<384>, 0, 1, s, what, a);
  return launch(k_norm_bwd<512, 2, WIDE>, b.blocks, kNormBackThreads<512>, 0, 1, s, what, a);
}

int clear(void* p, int64_t bytes, cudaStream_t s) {
  if (p == nullptr || bytes == 0) return GWS_OK;
  const cudaError_t err = cudaMemsetAsync(p, 0, static_cast<size_t>(bytes), s);
  return err == cudaSuccess ? GWS_OK : gws::report_cuda(err, "clearing a gradient");
}

// ---- AdamW -------------------------------------------------------------------------------------------------------------
int64_t moment_bytes(const gws_adamw_state& s) { return 2 * s.total * (s.format == GWS_ADAMW_8BIT ? 1 : 4); }

// Whether any output overlaps another one or an input: spans in the order of their addresses, the outputs' and everyone's farthest end so far.
struct Use {
  uintptr_t begin, end;
  bool written;
};
bool any_clash(std::vector<Use>& uses) {
  std::sort(uses.begin(), uses.end(), [](const Use& a, const Use& b) { return a.begin < b.begin; });
  uintptr_t all = 0, written = 0;
  for (const Use& u : uses) {
    if (u.begin == u.end) continue;
    if (u.begin < (u.written ? all : written)) return true;
    all = std::max(all, u.end);
    if (u.written) written = std::max(written, u.end);
  }
  return false;
}

template <int CAP>
int launch_adamw(const AdamwArgs& args, const AdamwRec* recs, int n, unsigned blocks, int format, cudaStream_t s) {
  AdamwBatch<CAP> b;
  b.a = args;
  b.a.n = n;
  std::memcpy(b.e, recs, sizeof(AdamwRec) * static_cast<size_t>(n));
  std::memset(b.e + n, 0, sizeof(AdamwRec) * static_cast<size_t>(CAP - n));
  bool loose = false;
  for (int i = 0; i < n; ++i) loose = loose || (recs[i].flags & (kAdamwWide | kAdamwF32)) == 0u;
  auto kernel = format == GWS_ADAMW_F32 ? k_adamw<GWS_ADAMW_F32, false, CAP> : loose ? k_adamw<GWS_ADAMW_8BIT, true, CAP> : k_adamw<GWS_ADAMW_8BIT, false, CAP>;
  return launch(kernel, blocks, 256, 0, 1, s, "AdamW kernel", b);
}

// Records of a launch: few tensors travel in 0.7 KB of kernel parameters, many in 15.
constexpr int kAdamwFew = 16, kAdamwMany = 384;

// `launches`: false for the checks alone.
int adamw_step(int n_tensors, void* const* params, const void* const* grads, const int64_t* sizes, const int64_t* starts, const int32_t* types, const double* decays,
               const gws_adamw_state* state, const gws_adamw_step_args* args, bool launches, cudaStream_t s) {
  if (n_tensors < 0) return GWS_ERR_SHAPE;
  if (state == nullptr || args == nullptr) return GWS_ERR_NULL;
  if (state->format != GWS_ADAMW_F32 && state->format != GWS_ADAMW_8BIT) return GWS_ERR_UNSUPPORTED;
  if (state->total < 0 || state->total % kAdamwGroup != 0 || (args->step_dev == nullptr && args->step < 1)) return GWS_ERR_SHAPE;
  if (state->total / kAdamwGroup > 0x7FFFFFFFLL) return GWS_ERR_LIMIT;
  if (!(args->beta1 >= 0.0 && args->beta1 < 1.0 && args->beta2 >= 0.0 && args->beta2 < 1.0 && args->eps >= 0.0)) return GWS_ERR_UNSUPPORTED;
  const bool device = args->lr_dev != nullptr || args->step_dev != nullptr;
  if (n_tensors == 0) return GWS_OK;
  if (params == nullptr || grads == nullptr || sizes == nullptr || starts == nullptr || types == nullptr || decays == nullptr) return GWS_ERR_NULL;
  std::vector<Use> uses;
  std::vector<AdamwRec> recs;
  uses.reserve(static_cast<size_t>(n_tensors) * 2 + 8);
  recs.reserve(static_cast<size_t>(n_tensors));
  auto use = [&](const void* p, int64_t bytes, bool written) {
    if (p != nullptr && bytes > 0) uses.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + static_cast<uintptr_t>(bytes), written});
  };
  std::vector<Use> places;                       // of the tensors in the state
  bool ordered = true;
  places.reserve(static_cast<size_t>(n_tensors));
  for (int i = 0; i < n_tensors; ++i) {
    if (grads[i] == nullptr || sizes[i] == 0) continue;
    if (params[i] == nullptr) return GWS_ERR_NULL;
    if (types[i] != GWS_TYPE_BF16 && types[i] != GWS_TYPE_F32) return GWS_ERR_UNSUPPORTED;
    const int64_t n = sizes[i], each = types[i] == GWS_TYPE_F32 ? 4 : 2;
    if (n < 0 || starts[i] < 0 || starts[i] % kAdamwGroup != 0 || n > state->total || starts[i] > state->total - round_up(n, kAdamwGroup)) return GWS_ERR_SHAPE;
    if (!on(params[i], static_cast<size_t>(each)) || !on(grads[i], static_cast<size_t>(each))) return GWS_ERR_ALIGN;
    use(params[i], n * each, true);
    use(grads[i], n * each, false);
    const uintptr_t at = static_cast<uintptr_t>(starts[i]);
    ordered = ordered && (places.empty() || at >= places.back().end);
    places.push_back({at, at + static_cast<uintptr_t>(round_up(n, kAdamwGroup)), true});
    const size_t boundary = static_cast<size_t>(each) * 8;
    AdamwRec r;
    r.p = params[i];
    r.g = grads[i];
    r.n = n;
    r.group0 = static_cast<uint32_t>(starts[i] / kAdamwGroup);
    r.block0 = 0;
    r.decay = static_cast<float>(device ? decays[i] : 1.0 - args->lr * decays[i]);
    r.flags = (each == 4 ? kAdamwF32 : 0u) | (on(params[i], boundary) && on(grads[i], boundary) ? kAdamwWide : 0u);
    recs.push_back(r);
  }
  if (recs.empty()) return GWS_OK;
  const bool bits8 = state->format == GWS_ADAMW_8BIT;
  if (state->moments == nullptr || (bits8 && state->units == nullptr) || (device && launches && args->scalars == nullptr)) return GWS_ERR_NULL;
  if (!on(state->moments, 32) || !on(state->units, 4) || !on(state->rest, 16) || !on(args->grad_scale, 4) || !on(args->lr_dev, 4) || !on(args->step_dev, 8) ||
      !on(args->scalars, 4))
    return GWS_ERR_ALIGN;
  if (!ordered && any_clash(places)) return GWS_ERR_ALIAS;
  use(state->moments, moment_bytes(*state), true);
  if (bits8) use(state->units, 2 * state->total / kAdamwGroup * 4, true);
  use(state->rest, state->total * 2, true);
  use(args->grad_scale, 4, false);
  use(args->lr_dev, 4, false);
  use(args->step_dev, 8, false);
  if (device) use(args->scalars, 12, true);
  if (any_clash(uses)) return GWS_ERR_ALIAS;
  if (!launches) return GWS_OK;

  AdamwArgs a;
  std::memset(&a, 0, sizeof a);
  a.codes = static_cast<uint8_t*>(state->moments);
  a.units = state->units;
  a.rest = static_cast<int16_t*>(state->rest);
  a.total = state->total;
  a.grad_scale = args->grad_scale;
  a.b1 = static_cast<float>(args->beta1);
  a.to_m = static_cast<float>(1.0 - args->beta1);
  a.b2 = static_cast<float>(args->beta2);
  a.to_v = static_cast<float>(1.0 - args->beta2);
  a.eps = static_cast<float>(args->eps);
  if (device) {
    a.scalars = args->scalars;
    const int st = launch(k_adamw_scalars, 1, 1, 0, 1, s, "AdamW scalars kernel", args->step_dev, args->lr_dev, args->step, args->lr, args->beta1, args->beta2, args->scalars);
    if (st != GWS_OK) return st;
  } else {
    a.alpha = static_cast<float>(args->lr / (1.0 - std::pow(args->beta1, static_cast<double>(args->step))));
    a.rho = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(args->beta2, static_cast<double>(args->step))));
  }
  // Few groups: one to a warp, so that every SM has its share.  Many: eight to a warp, which finds its tensor once for all of them.
  int64_t groups = 0;
  for (const AdamwRec& r : recs) groups += (r.n + kAdamwGroup - 1) / kAdamwGroup;
  a.per = groups >= 8 * 64 * 148 ? 64u : groups >= 2 * 16 * 148 ? 16u : 8u;
  for (size_t first = 0; first < recs.size();) {
    int n = 0;
    int64_t blocks = 0;
    for (; first + n < recs.size() && n < kAdamwMany; ++n) {
      AdamwRec& r = recs[first + n];
      const int64_t more = (r.n + a.per * static_cast<int64_t>(kAdamwGroup) - 1) / (a.per * static_cast<int64_t>(kAdamwGroup));
      if (blocks + more > 0x7FFFFFFFLL) break;
      r.block0 = static_cast<uint32_t>(blocks);
      blocks += more;
    }
    const int st = n <= kAdamwFew ? launch_adamw<kAdamwFew>(a, recs.data() + first, n, static_cast<unsigned>(blocks), state->format, s)
                                  : launch_adamw<kAdamwMany>(a, recs.data() + first, n, static_cast<unsigned>(blocks), state->format, s);
    if (st != GWS_OK) return st;
    first += static_cast<size_t>(n);
  }
  return GWS_OK;
}

}  // namespace

extern "C" {

int64_t gws_layernorm_workspace_bytes(const gws_norm_desc* desc) {
  const int st = check_norm(desc);
  if (st != GWS_OK) return st;
  if (desc->rows == 0 || desc->cols == 0) return 0;
  return round_up(static_cast<int64_t>(norm_back(desc->rows, desc->cols).blocks) * 2 * desc->cols * 4, 256);
}

int gws_layernorm_fwd(const gws_norm_desc* desc, const void* x, const void* residual, const void* weight, const void* bias, void* y, void* sum, float* stats,
                      void* stream) {
  const int st = check_norm(desc);
  if (st != GWS_OK) return st;
  const gws_norm_desc& d = *desc;
  if (bias != nullptr && weight == nullptr) return GWS_ERR_UNSUPPORTED;
  if (d.rows == 0 || d.cols == 0) return GWS_OK;
  if ((d.rows > 1 && d.ld_x < d.cols) || (d.rows > 1 && residual != nullptr && d.ld_residual < d.cols)) return GWS_ERR_SHAPE;
  if (x == nullptr || y == nullptr || (residual != nullptr && sum == nullptr)) return GWS_ERR_NULL;
  const size_t wb = static_cast<size_t>(weight_bytes(d));
  if (!on(x, 2) || !on(residual, 2) || !on(y, 2) || !on(sum, 2) || !on(weight, wb) || !on(bias, wb) || !on(stats, 4)) return GWS_ERR_ALIGN;
  const int64_t vector = d.cols * weight_bytes(d);
  if (clash({rows_of(y, d.rows, d.cols, d.cols), rows_of(residual != nullptr ? sum : nullptr, d.rows, d.cols, d.cols), {stats, stats != nullptr ? d.rows * 8 : 0}},
            {rows_of(x, d.rows, d.cols, d.ld_x), rows_of(residual, d.rows, d.cols, d.ld_residual), {weight, weight != nullptr ? vector : 0},
             {bias, bias != nullptr ? vector : 0}}))
    return GWS_ERR_ALIAS;
  NormArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = static_cast<const uint16_t*>(x);
  a.r = static_cast<const uint16_t*>(residual);
  a.ld_x = d.ld_x;
  a.ld_r = d.ld_residual;
  a.weight = weight;
  a.bias = bias;
  a.y = static_cast<uint16_t*>(y);
  a.sum = static_cast<uint16_t*>(sum);
  a.stats = stats;
  a.rows = d.rows;
  a.cols = d.cols;
  a.eps = d.eps;
  a.f32 = d.weight_type == GWS_TYPE_F32;
  const bool wide = d.cols % 8 == 0 && wide_rows(x, d.rows, d.ld_x) && wide_rows(residual, d.rows, d.ld_residual) && on(y, 16) && (residual == nullptr || on(sum, 16)) &&
                    on(weight, 16) && on(bias, 16);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return wide ? launch_norm_fwd<true>(a, s) : launch_norm_fwd<false>(a, s);
}

int gws_layernorm_bwd(const gws_norm_desc* desc, const void* grad_y, const void* s_in, const void* weight, const float* stats, const void* grad_sum, void* grad_x,
                      void* grad_weight, void* grad_bias, void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_norm(desc);
  if (st != GWS_OK) return st;
  const gws_norm_desc& d = *desc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const size_t wb = static_cast<size_t>(weight_bytes(d));
  if (!on(grad_x, 2) || !on(grad_weight, wb) || !on(grad_bias, wb)) return GWS_ERR_ALIGN;
  if (d.rows == 0 || d.cols == 0) {
    if ((st = clear(grad_weight, d.cols * weight_bytes(d), s)) != GWS_OK) return st;
    return clear(grad_bias, d.cols * weight_bytes(d), s);
  }
  if (d.rows > 1 && (d.ld_x < d.cols || d.ld_grad_y < d.cols || (grad_sum != nullptr && d.ld_grad_sum < d.cols))) return GWS_ERR_SHAPE;
  const bool sums = grad_weight != nullptr || grad_bias != nullptr;
  if (!sums && grad_x == nullptr) return GWS_OK;
  if (grad_y == nullptr || s_in == nullptr || stats == nullptr) return GWS_ERR_NULL;
  if (!on(grad_y, 2) || !on(s_in, 2) || !on(weight, wb) || !on(stats, 4) || !on(grad_sum, 2)) return GWS_ERR_ALIGN;
  const NormBack b = norm_back(d.rows, d.cols);
  const int64_t vector = d.cols * weight_bytes(d), need = sums ? gws_layernorm_workspace_bytes(desc) : 0;
  if (clash({rows_of(grad_x, d.rows, d.cols, d.cols), {grad_weight, grad_weight != nullptr ? vector : 0}, {grad_bias, grad_bias != nullptr ? vector : 0},
             {workspace, workspace != nullptr ? need : 0}},
            {rows_of(grad_y, d.rows, d.cols, d.ld_grad_y), rows_of(s_in, d.rows, d.cols, d.ld_x), rows_of(grad_sum, d.rows, d.cols, d.ld_grad_sum),
             {weight, weight != nullptr ? vector : 0}, {stats, d.rows * 8}}))
    return GWS_ERR_ALIAS;
  if (!workspace_ok(workspace, workspace_bytes, need)) return GWS_ERR_WORKSPACE;
  NormArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = static_cast<const uint16_t*>(s_in);
  a.dy = static_cast<const uint16_t*>(grad_y);
  a.d = grad_x != nullptr ? static_cast<const uint16_t*>(grad_sum) : nullptr;
  a.ld_x = d.ld_x;
  a.ld_dy = d.ld_grad_y;
  a.ld_d = d.ld_grad_sum;
  a.weight = weight;
  a.dx = static_cast<uint16_t*>(grad_x);
  a.stats = const_cast<float*>(stats);
  a.part = sums ? static_cast<float*>(workspace) : nullptr;
  a.rows = d.rows;
  a.cols = d.cols;
  a.eps = d.eps;
  a.f32 = d.weight_type == GWS_TYPE_F32;
  if (b.team == 0) {
    if (grad_x != nullptr && (st = launch(k_norm_bwd_long, static_cast<unsigned>(d.rows), kNormLong, 0, 1, s, "layer norm backward kernel", a)) != GWS_OK) return st;
    if (sums && (st = launch(k_norm_columns, blocks_for(d.cols, 256) * b.blocks, 256, 0, 1, s, "layer norm column sums", a, b.blocks)) != GWS_OK) return st;
  } else {
    const bool wide = d.cols % 8 == 0 && wide_rows(grad_y, d.rows, d.ld_grad_y) && wide_rows(s_in, d.rows, d.ld_x) && wide_rows(a.d, d.rows, d.ld_grad_sum) &&
                      on(weight, 16) && on(grad_x, 16);
    if ((st = wide ? launch_norm_bwd<true>(a, b, s) : launch_norm_bwd<false>(a, b, s)) != GWS_OK) return st;
  }
  if (!sums) return GWS_OK;
  return launch(k_column_sums, blocks_for(d.cols, 32) * 2u, 32 * kSumWarps, 0, 1, s, "join of column sums", static_cast<const float*>(a.part), b.blocks, d.cols, 2u, grad_weight,
                grad_bias, a.f32);
}

int gws_adamw_step(int n_tensors, void* const* params, const void* const* grads, const int64_t* sizes, const int64_t* starts, const int32_t* types,
                   const double* weight_decay, const gws_adamw_state* state, const gws_adamw_step_args* args, void* stream) {
  try {
    return adamw_step(n_tensors, params, grads, sizes, starts, types, weight_decay, state, args, true, static_cast<cudaStream_t>(stream));
  } catch (...) {                      // host memory for the list of tensors
    return GWS_ERR_LIMIT;
  }
}

int gws_adamw_check(int n_tensors, void* const* params, const void* const* grads, const int64_t* sizes, const int64_t* starts, const int32_t* types,
                    const double* weight_decay, const gws_adamw_state* state, const gws_adamw_step_args* args) {
  try {
    return adamw_step(n_tensors, params, grads, sizes, starts, types, weight_decay, state, args, false, nullptr);
  } catch (...) {
    return GWS_ERR_LIMIT;
  }
}

int gws_adamw_values(const gws_adamw_state* state, float* m, float* v, void* stream) {
  if (state == nullptr) return GWS_ERR_NULL;
  if (state->format != GWS_ADAMW_8BIT) return GWS_ERR_UNSUPPORTED;
  if (state->total < 0 || state->total % kAdamwGroup != 0) return GWS_ERR_SHAPE;
  if (state->total / kAdamwGroup > 0x7FFFFFFFLL) return GWS_ERR_LIMIT;
  if (state->total == 0) return GWS_OK;
  if (state->moments == nullptr || state->units == nullptr || m == nullptr || v == nullptr) return GWS_ERR_NULL;
  if (!on(state->moments, 32) || !on(state->units, 4) || !on(m, 32) || !on(v, 32)) return GWS_ERR_ALIGN;
  const int64_t bytes = state->total * 4;
  if (clash({{m, bytes}, {v, bytes}}, {{state->moments, moment_bytes(*state)}, {state->units, 2 * state->total / kAdamwGroup * 4}})) return GWS_ERR_ALIAS;
  return launch(k_adamw_values, blocks_for(state->total, 2048), 256, 0, 1, static_cast<cudaStream_t>(stream), "AdamW values kernel",
                static_cast<const uint8_t*>(state->moments), static_cast<const float*>(state->units), state->total, m, v);
}

}  // extern "C"
