// Host logic of include/lite_attn_layer.h (no HIP call, no device code): argument checks, and how a call is laid out on the
// chip.  Also builds with a plain C++ compiler under the CPU sanitizers.
#include "lite_attn_layer_kernels.h"

#include <algorithm>
#include <cmath>

#include "lite_attn_kernels.h"

namespace la {

namespace {

constexpr int kCUs = 256;
constexpr int64_t kMaxRows = (int64_t)1 << 30;  // of a call: row and token numbers stay within quotient()'s range

int size_of(int dtype) { return dtype == LITE_ATTN_F32 ? 4 : 2; }
bool known(int dtype) { return dtype >= LITE_ATTN_BF16 && dtype <= LITE_ATTN_F32; }
bool good_eps(float eps) { return eps >= 0.f && std::isfinite(eps); }
size_t up16(size_t x) { return (x + 15) & ~(size_t)15; }

// A tensor of `n` axes (sizes, strides over them, elements) and a last one of `inner` contiguous elements.
struct View {
  const void* data;
  int n;
  int64_t size[3], stride[3], inner;
  int dtype;
};

View view(const lite_attn_heads_t& t, const lite_attn_rotary_desc_t& d, int heads) {
  return {t.data, 3, {d.batch, heads, d.seqlen}, {t.stride_b, t.stride_h, t.stride_n}, d.head_dim, d.dtype};
}
View view(const lite_attn_rows_t& t, int batch, int rows, int dim, int dtype) {
  return {t.data, 2, {batch, rows, 0}, {t.stride_b, t.stride_n, 0}, dim, dtype};
}

// Aligned to its type, strides not negative, its extent within an address; a result has no two elements in one place: each
// axis steps over all of the axes with smaller strides.
bool good(const View& v, bool result) {
  for (int x = 0; x < v.n; ++x)
    if (v.size[x] == 0) return true;  // nothing there, of which the address need not be one
  if (!v.data || ((uintptr_t)v.data & (size_of(v.dtype) - 1))) return false;
  constexpr int64_t kMost = (int64_t)1 << 46;  // elements
  int64_t extent = v.inner;
  int order[3] = {0, 1, 2};
  std::sort(order, order + v.n, [&](int a, int b) { return v.stride[a] < v.stride[b]; });
  for (int x = 0; x < v.n; ++x) {
    const int64_t size = v.size[order[x]], stride = v.stride[order[x]];
    if (size <= 1) continue;
    if (stride < (result ? extent : 0) || stride > kMost) return false;
    if (stride > kMost / (size - 1)) return false;
    extent += stride * (size - 1);
    if (extent > kMost) return false;
  }
  return true;
}

template <class T>
bool good_vector(const T* p, int dtype) {
  return ((uintptr_t)p & (size_of(dtype) - 1)) == 0;
}
bool good_grad(const float* p) { return ((uintptr_t)p & 3) == 0; }

// Shares that each of `kinds` kinds of rows is dealt to, at most `rows` (of a kind), in workgroups of `waves` waves, `per_cu`
// of them on a CU.  A workgroup has a row asked for at any time, and memory gives most when some 15 to 18 KB are asked for on
// each CU, in whole workgroups for each CU: more of them get into each other's way, fewer do not keep it busy.  us at 256 /
// 512 / 768 / 1024 / 1280 / 1536 workgroups: forwards 32760 x 1536, 9 KB a row, 114 / 104 / 111 / 111 / 113 / 114, 60000 x
// 1111, 4 KB, - / - / 108 / 115 / 124 / 127, 75600 x 5120, 20 KB, 514 / 564 / 555 / 592 / 614 / 607, backwards 32760 x 1536,
// 18 KB, 158 / 169 / 189 / 191 / 198 / 207, 12 KB, 149 / 119 / 128 / 136 / 148 / 154, rotary of 12 heads, 3 KB, 167 / 109 /
// 87 / 83 / 81 / 81, backwards, 6 KB, 220 / 138 / 116 / 121 / 119 / 118.  Kinds that do not go evenly into that are dealt to
// four times as many, to be taken as CUs get free.
int shares_of(int64_t kinds, int rows, int waves, int64_t per_cu) {
  const int64_t side_by_side = kCUs * std::max<int64_t>(1, std::min<int64_t>(per_cu, 32 / waves));
  const int64_t shares = kinds * 4 <= side_by_side ? side_by_side / kinds : (4 * side_by_side + kinds - 1) / kinds;
  return (int)std::max<int64_t>(1, std::min<int64_t>(rows, shares));
}

int launch_of(int64_t kinds, int64_t shares, int threads, LayerLaunch* l) {
  if (kinds * shares * threads >= (int64_t)1 << 32) return LITE_ATTN_EUNSUPPORTED;  // (what a launch may have)
  l->threads = threads;
  l->blocks = (int)(kinds * shares);
  return LITE_ATTN_OK;
}

int log2_up(int x) {
  int l = 0;
  while ((1 << l) < x) ++l;
  return l;
}

struct RotaryShape {
  int lanes, team_heads, near_heads, groups, row_lanes, sum_log, tokens, threads, shares;
  Sums sums;
  int kinds;  // of workgroups of a batch entry
};

// How the tokens of a call may be taken: one by one, or several neighbouring ones, which must not lie too far apart; heads-first,
// forwards, if these are neighbours in a result too.
enum Taken { kOneByOne, kTogether, kHeadsFirst };

// A head takes a thread for each kEach entries; a workgroup takes all heads of a token (NORM_ROW) or an even part of them, and,
// where these are few, several tokens: us with a token in a workgroup of its own -> with 8 tokens, 302400 tokens of 2 heads of
// 128 153 -> 115, backwards through a norm 376 -> 197; 2 x 3913 tokens of 5 heads of 72, backwards, 27.6 -> 24.9.
// The part is what 256 threads hold; for results that are heads-first a quarter of that, so that there are four tokens or more
// and what is written lies side by side in longer runs: us at 75600 tokens of 24 heads of 128 369 -> 337, of 64 195 -> 184, 20 of
// 80 281 -> 205, 12 of 96 185 -> 146, 37 of 72 504 -> 372 (32 bits, 12 of 72 227 -> 234).  (Backwards the sums for the weights'
// gradient would come in another order.)  And a smaller part where fewer than 0.72 of its threads have an entry and one more
// split or a few give 0.9: 30 heads of 72 347 -> 280, 24 of 88 320 -> 252, backwards the same; from 0.75 to 0.98, 16 of 72, it is
// 147 -> 151.
RotaryShape rotary_shape(const lite_attn_rotary_desc_t& d, bool bwd, Taken taken) {
  RotaryShape s;
  const bool by_row = d.norm == LITE_ATTN_NORM_ROW;
  const int most = std::max(d.heads_q, d.heads_k);
  s.lanes = (d.head_dim + kEach - 1) / kEach;
  const int room = by_row ? most : std::max(1, (taken == kHeadsFirst ? 64 : 256) / s.lanes);
  s.groups = (most + room - 1) / room;
  if (!by_row && taken == kTogether) {
    auto in_use = [&](int groups) {
      const int row = (most + groups - 1) / groups * s.lanes, tokens = std::max(1, 256 / row);
      return (double)most * s.lanes * tokens / (groups * ((tokens * row + 63) / 64 * 64));
    };
    for (int g = s.groups + 1; in_use(s.groups) < 0.72 && g <= std::min(most, s.groups + 4); ++g)
      if (in_use(g) >= 0.9) s.groups = g;
  }
  s.team_heads = (most + s.groups - 1) / s.groups;
  s.groups = (most + s.team_heads - 1) / s.team_heads;
  s.row_lanes = s.team_heads * s.lanes;
  s.sum_log = 0;
  if (d.norm == LITE_ATTN_NORM_NONE) {
    s.sums = kSumNone;
  } else if (by_row && s.row_lanes <= 64) {
    s.sums = kSumLanes;
    s.sum_log = log2_up(s.row_lanes);
    s.row_lanes = 1 << s.sum_log;
  } else if (by_row) {
    s.sums = kSumWaves;
  } else if ((s.lanes & (s.lanes - 1)) == 0) {
    s.sums = kSumLanes;
    s.sum_log = log2_up(s.lanes);
  } else {
    s.sums = kSumHeads;
  }
  s.tokens = taken != kOneByOne && s.sums != kSumWaves ? std::max(1, std::min(256 / s.row_lanes, d.seqlen)) : 1;
  s.threads = (s.tokens * s.row_lanes + 63) / 64 * 64;
  s.near_heads = s.tokens > 1 ? s.team_heads : std::min(s.team_heads, 64 % s.lanes ? 63 / s.lanes + 2 : 64 / s.lanes);
  s.kinds = s.groups * (rotary_sides(d.norm != LITE_ATTN_NORM_NONE, bwd) == 1 && d.heads_k ? 2 : 1);
  const int64_t bytes = (int64_t)s.tokens * s.team_heads * d.head_dim * size_of(d.dtype) *
                        (bwd && d.norm != LITE_ATTN_NORM_NONE ? 2 : 1);
  s.shares = shares_of((int64_t)d.batch * s.kinds, (int)(((int64_t)d.seqlen + s.tokens - 1) / s.tokens), s.threads / 64,
                       (18432 + bytes - 1) / bytes);
  return s;
}

// Whether neighbouring tokens of a head lie next to each other.
bool heads_first(const lite_attn_heads_t& t) { return t.stride_n < t.stride_h; }

// Whether what a workgroup (a wave, if it takes one token at a time) has of a tensor lies within 4 GiB: offsets have 32 bits.
bool near(const lite_attn_heads_t& t, const lite_attn_rotary_desc_t& d, const RotaryShape& s, int heads) {
  const int apart = std::min(heads, s.near_heads) - 1;
  const int64_t most = (((int64_t)1 << 32) - 4096) / size_of(d.dtype) - d.head_dim;
  if (apart > 0 && t.stride_h > most / apart) return false;
  const int64_t left = most - (apart > 0 ? apart * t.stride_h : 0);
  return s.tokens == 1 || t.stride_n <= left / (s.tokens - 1);
}

// Floats that one share leaves for the weights' gradient of a side.
size_t rotary_part(const lite_attn_rotary_desc_t& d, const RotaryShape& s, int side) {
  const int heads = side ? d.heads_k : d.heads_q;
  return (size_t)(d.norm == LITE_ATTN_NORM_ROW ? s.tokens * heads : heads ? s.groups : 0) * d.head_dim;
}
size_t rotary_workspace(const lite_attn_rotary_desc_t& d, const RotaryShape& s) {
  return up16(sizeof(float) * d.batch * s.shares * (rotary_part(d, s, 0) + rotary_part(d, s, 1)));
}

int fill_rotary(const lite_attn_rotary_desc_t& d, const lite_attn_positions_t& at, const void* const weights[2],
                const RotaryShape& s, RotaryParams* p) {
  *p = RotaryParams();
  if (d.pairs > 0 && (!at.freqs || ((uintptr_t)at.freqs & 7))) return LITE_ATTN_EINVAL;
  if (at.positions) {
    if (((uintptr_t)at.positions & 3) || at.positions_stride_b < 0 || at.positions_stride_b > ((int64_t)1 << 46))
      return LITE_ATTN_EINVAL;
  } else if (at.token_start < 0 || (int64_t)at.token_start + d.seqlen > kMaxRows) {
    return LITE_ATTN_EINVAL;
  }
  for (int x = 0; x < 2; ++x) {
    if (weights[x] && d.norm == LITE_ATTN_NORM_NONE) return LITE_ATTN_EINVAL;
    if (!good_vector(weights[x], d.weight_dtype)) return LITE_ATTN_EINVAL;
    p->side[x].w = weights[x];
    p->side[x].heads = x ? d.heads_k : d.heads_q;
    p->side[x].inv_count = 1.f / (float)(d.head_dim * (d.norm == LITE_ATTN_NORM_ROW ? std::max(1, p->side[x].heads) : 1));
  }
  p->freqs = at.freqs;
  p->positions = at.positions;
  p->positions_stride_b = at.positions_stride_b;
  p->sides = d.heads_k ? 2 : 1;
  p->batch = d.batch;
  p->N = d.seqlen;
  p->tokens = s.tokens;
  p->shares = s.shares;
  p->head_dim = d.head_dim;
  p->pairs = d.pairs;
  p->lanes = s.lanes;
  p->team_heads = s.team_heads;
  p->groups = s.groups;
  p->near_heads = s.near_heads;
  p->row_lanes = s.row_lanes;
  p->sum_log = s.sum_log;
  p->by_row = d.norm == LITE_ATTN_NORM_ROW;
  p->halves = d.halves;
  p->weight_dtype = d.weight_dtype;
  p->token_start = at.token_start;
  p->area = d.grid[1] * d.grid[2];
  p->width = d.grid[2];
  p->video = d.grid[0] * p->area;
  p->eps = d.eps;
  p->per_area = reciprocal(p->area);
  p->per_width = reciprocal(p->width);
  p->per_lanes = reciprocal(s.lanes);
  p->per_row = reciprocal(s.row_lanes);
  p->per_tokens = reciprocal(s.tokens);
  p->per_angles = reciprocal(4 * s.lanes);
  return LITE_ATTN_OK;
}

// Whether the entries of neighbouring tokens share a line of memory.
bool shares_lines(const lite_attn_heads_t& t, const lite_attn_rotary_desc_t& d) {
  return t.stride_n * size_of(d.dtype) % 128 != 0;
}

void set(int64_t to[3], const lite_attn_heads_t& t, int dtype) {
  to[0] = t.stride_b * size_of(dtype);
  to[1] = t.stride_h * size_of(dtype);
  to[2] = t.stride_n * size_of(dtype);
}
Lines lines(const lite_attn_rows_t& t, int dtype) {
  return {static_cast<char*>(t.data), t.stride_b * size_of(dtype), t.stride_n * size_of(dtype)};
}

}  // namespace

int check_rotary(const lite_attn_rotary_desc_t* d) {
  if (!d) return LITE_ATTN_EINVAL;
  if (d->batch < 1 || d->seqlen < 0 || d->heads_q < 1 || d->heads_k < 0 || d->head_dim < 2 || d->head_dim % 2)
    return LITE_ATTN_EINVAL;
  if (!known(d->dtype) || !known(d->weight_dtype)) return LITE_ATTN_EINVAL;
  if (d->norm != LITE_ATTN_NORM_NONE && d->norm != LITE_ATTN_NORM_HEAD && d->norm != LITE_ATTN_NORM_ROW)
    return LITE_ATTN_EINVAL;
  if ((d->halves != 0 && d->halves != 1) || d->pairs < 0 || d->pairs > d->head_dim / 2) return LITE_ATTN_EINVAL;
  if (d->grid[0] < 1 || d->grid[1] < 1 || d->grid[2] < 1 || !good_eps(d->eps)) return LITE_ATTN_EINVAL;
  if (d->head_dim > 512) return LITE_ATTN_EUNSUPPORTED;
  const int64_t lanes = (d->head_dim + kEach - 1) / kEach, most = std::max(d->heads_q, d->heads_k);
  if (d->norm == LITE_ATTN_NORM_ROW && most * lanes > kMaxTeam) return LITE_ATTN_EUNSUPPORTED;
  if (most > 1 << 16) return LITE_ATTN_EUNSUPPORTED;
  if ((int64_t)d->batch * d->seqlen > kMaxRows) return LITE_ATTN_EUNSUPPORTED;
  const int64_t area = (int64_t)d->grid[1] * d->grid[2];
  if (area > kMaxRows || area * d->grid[0] > kMaxRows) return LITE_ATTN_EUNSUPPORTED;
  return LITE_ATTN_OK;
}

int plan_rotary(const lite_attn_rotary_desc_t& d, const lite_attn_rotary_fwd_t& a, RotaryParams* p, LayerLaunch* l) {
  const int heads[2] = {d.heads_q, d.heads_k}, sides = d.heads_k ? 2 : 1;
  const lite_attn_heads_t in[2] = {a.q, a.k}, out[2] = {a.q_out, a.k_out};
  const bool first = heads_first(out[0]) || (sides == 2 && heads_first(out[1]));
  RotaryShape s = rotary_shape(d, false, first ? kHeadsFirst : kTogether);
  for (int x = 0; x < sides; ++x) {
    if (!good(view(in[x], d, heads[x]), false) || !good(view(out[x], d, heads[x]), true)) return LITE_ATTN_EINVAL;
    if (!near(in[x], d, s, heads[x]) || !near(out[x], d, s, heads[x])) s = rotary_shape(d, false, kOneByOne);
  }
  for (int x = 0; x < sides; ++x)
    if (!near(in[x], d, s, heads[x]) || !near(out[x], d, s, heads[x])) return LITE_ATTN_EUNSUPPORTED;
  const void* const weights[2] = {a.q_weight, a.k_weight};
  const int rc = fill_rotary(d, a.at, weights, s, p);
  if (rc != LITE_ATTN_OK) return rc;
  for (int x = 0; x < sides; ++x) {
    p->side[x].x = static_cast<const char*>(in[x].data);
    p->side[x].out = static_cast<char*>(out[x].data);
    set(p->side[x].xs, in[x], d.dtype);
    set(p->side[x].os, out[x], d.dtype);
    p->shared_writes |= shares_lines(out[x], d);
    p->shared_reads |= p->shared_writes | shares_lines(in[x], d);
  }
  l->sums = s.sums;
  return launch_of(d.batch, (int64_t)s.shares * s.kinds, s.threads, l);
}

int plan_rotary(const lite_attn_rotary_desc_t& d, const lite_attn_rotary_bwd_t& a, RotaryParams* p, LayerLaunch* l) {
  const int heads[2] = {d.heads_q, d.heads_k}, sides = d.heads_k ? 2 : 1;
  const lite_attn_heads_t in[2] = {a.q, a.k}, g[2] = {a.dq_out, a.dk_out}, out[2] = {a.dq, a.dk};
  float* const grads[2] = {a.dq_weight, a.dk_weight};
  const bool normed = d.norm != LITE_ATTN_NORM_NONE;
  RotaryShape s = rotary_shape(d, true, kTogether);
  auto all_near = [&](int x) {
    return (!normed || near(in[x], d, s, heads[x])) && near(g[x], d, s, heads[x]) && near(out[x], d, s, heads[x]);
  };
  for (int x = 0; x < sides; ++x) {
    if (normed && !good(view(in[x], d, heads[x]), false)) return LITE_ATTN_EINVAL;
    if (!good(view(g[x], d, heads[x]), false) || !good(view(out[x], d, heads[x]), true)) return LITE_ATTN_EINVAL;
    if (!all_near(x)) s = rotary_shape(d, true, kOneByOne);
  }
  for (int x = 0; x < sides; ++x)
    if (!all_near(x)) return LITE_ATTN_EUNSUPPORTED;
  const void* const weights[2] = {a.q_weight, a.k_weight};
  const int rc = fill_rotary(d, a.at, weights, s, p);
  if (rc != LITE_ATTN_OK) return rc;
  if (!normed && (grads[0] || grads[1])) return LITE_ATTN_EINVAL;
  if (!good_grad(grads[0]) || !good_grad(grads[1])) return LITE_ATTN_EINVAL;
  if (grads[0] || grads[1]) {
    if (a.workspace_bytes < lite_attn_rotary_bwd_workspace(&d) || !a.workspace || ((uintptr_t)a.workspace & 15))
      return LITE_ATTN_EWORKSPACE;
  }
  float* part = static_cast<float*>(a.workspace);
  for (int x = 0; x < sides; ++x) {
    p->side[x].x = static_cast<const char*>(in[x].data);
    p->side[x].g = static_cast<const char*>(g[x].data);
    p->side[x].out = static_cast<char*>(out[x].data);
    set(p->side[x].xs, in[x], d.dtype);
    set(p->side[x].gs, g[x], d.dtype);
    set(p->side[x].os, out[x], d.dtype);
    p->shared_writes |= shares_lines(out[x], d);
    p->shared_reads |= p->shared_writes | shares_lines(g[x], d) | (normed && shares_lines(in[x], d));
    if (grads[x]) p->side[x].part = part;
    part += (size_t)d.batch * s.shares * rotary_part(d, s, x);
  }
  l->sums = s.sums;
  return launch_of(d.batch, (int64_t)s.shares * s.kinds, s.threads, l);
}

namespace {

struct ResidualShape {
  int threads, shares;
};

int groups_of(const lite_attn_residual_desc_t& d) {
  return (int)(((int64_t)d.seqlen + d.tokens_per_mod - 1) / d.tokens_per_mod);
}

// A workgroup takes a row of `dim` entries, kEach in a thread, and rows of one group (tokens that share a row of modulation).
// Backwards through a norm of y, whose sums come one after the other, a row takes longer, and one more workgroup on a CU pays
// (us at 60000 x 1112, three -> four 207 -> 192; not in place of a single one, at 40000 x 5120 461 -> 480).
ResidualShape residual_shape(const lite_attn_residual_desc_t& d, bool bwd) {
  ResidualShape s;
  s.threads = (d.dim + 64 * kEach - 1) / (64 * kEach) * 64;
  const int64_t bytes = (int64_t)d.dim * (size_of(d.dtype) + size_of(d.stream_dtype));
  int64_t per_cu = bwd ? (18432 + 2 * bytes - 1) / (2 * bytes) : (14848 + bytes / 2) / bytes;
  if (bwd && d.post_norm != LITE_ATTN_NORM_NONE && per_cu > 1) ++per_cu;
  s.shares = shares_of(std::max<int64_t>(1, (int64_t)d.batch * groups_of(d)), std::min(d.tokens_per_mod, d.seqlen),
                       s.threads / 64, per_cu);
  return s;
}

// Rows of modulation, or none.
bool modulation(const lite_attn_rows_t& t, const lite_attn_residual_desc_t& d, Lines* to) {
  *to = lines(t, d.param_dtype);
  return !t.data || good(view(t, d.batch, groups_of(d), d.dim, d.param_dtype), false);
}

int fill_residual(const lite_attn_residual_desc_t& d, const ResidualShape& s, const lite_attn_rows_t& gate,
                  const lite_attn_rows_t& scale, const void* post_w, const void* pre_w, const void* pre_b,
                  ResidualParams* p) {
  *p = ResidualParams();
  if (!modulation(gate, d, &p->gate) || !modulation(scale, d, &p->scale)) return LITE_ATTN_EINVAL;
  for (const void* v : {post_w, pre_w, pre_b})
    if (!good_vector(v, d.param_dtype)) return LITE_ATTN_EINVAL;
  p->post_w = post_w;
  p->pre_w = pre_w;
  p->pre_b = pre_b;
  p->batch = d.batch;
  p->N = d.seqlen;
  p->D = d.dim;
  p->per_mod = std::min(d.tokens_per_mod, std::max(1, d.seqlen));
  p->groups = groups_of(d);
  p->shares = s.shares;
  p->post = d.post_norm;
  p->pre = d.pre_norm;
  p->param_dtype = d.param_dtype;
  p->post_eps = d.post_eps;
  p->pre_eps = d.pre_eps;
  p->alpha = d.residual_scale;
  p->inv_D = 1.f / (float)d.dim;
  return LITE_ATTN_OK;
}

}  // namespace

int check_residual(const lite_attn_residual_desc_t* d) {
  if (!d) return LITE_ATTN_EINVAL;
  if (d->batch < 1 || d->seqlen < 0 || d->dim < 1 || d->tokens_per_mod < 1) return LITE_ATTN_EINVAL;
  if (!known(d->dtype) || !known(d->stream_dtype) || !known(d->param_dtype)) return LITE_ATTN_EINVAL;
  for (const int norm : {d->post_norm, d->pre_norm})
    if (norm != LITE_ATTN_NORM_NONE && norm != LITE_ATTN_NORM_RMS && norm != LITE_ATTN_NORM_LAYER) return LITE_ATTN_EINVAL;
  if (!good_eps(d->post_eps) || !good_eps(d->pre_eps) || !std::isfinite(d->residual_scale)) return LITE_ATTN_EINVAL;
  if (d->stream_dtype != d->dtype && d->stream_dtype != LITE_ATTN_F32) return LITE_ATTN_EUNSUPPORTED;
  if (d->dim > kEach * kMaxTeam) return LITE_ATTN_EUNSUPPORTED;
  if ((int64_t)d->batch * d->seqlen > kMaxRows) return LITE_ATTN_EUNSUPPORTED;
  return LITE_ATTN_OK;
}

int plan_residual(const lite_attn_residual_desc_t& d, const lite_attn_residual_fwd_t& a, ResidualParams* p,
                  LayerLaunch* l) {
  const ResidualShape s = residual_shape(d, false);
  const int rc = fill_residual(d, s, a.gate, a.scale, a.post_weight, a.pre_weight, a.pre_bias, p);
  if (rc != LITE_ATTN_OK) return rc;
  if (!modulation(a.shift, d, &p->shift)) return LITE_ATTN_EINVAL;
  if (!a.x.data || (!a.x_out.data && !a.h.data)) return LITE_ATTN_EINVAL;
  auto take = [&](const lite_attn_rows_t& t, int dtype, bool result, Lines* to) {
    *to = lines(t, dtype);
    return !t.data || good(view(t, d.batch, d.seqlen, d.dim, dtype), result);
  };
  if (!take(a.x, d.stream_dtype, false, &p->x) || !take(a.y, d.dtype, false, &p->y) ||
      !take(a.x_out, d.stream_dtype, true, &p->x_out) || !take(a.h, d.dtype, true, &p->h))
    return LITE_ATTN_EINVAL;
  return launch_of((int64_t)d.batch * p->groups, s.shares, s.threads, l);
}

int plan_residual(const lite_attn_residual_desc_t& d, const lite_attn_residual_bwd_t& a, ResidualParams* p,
                  LayerLaunch* l) {
  const ResidualShape s = residual_shape(d, true);
  const int rc = fill_residual(d, s, a.gate, a.scale, a.post_weight, a.pre_weight, a.pre_bias, p);
  if (rc != LITE_ATTN_OK) return rc;
  const bool normed_y = d.post_norm != LITE_ATTN_NORM_NONE, normed_x = d.pre_norm != LITE_ATTN_NORM_NONE;
  if (d.seqlen > 0 && a.dh.data && !a.x_out.data && (normed_x || a.dscale || a.dpre_weight)) return LITE_ATTN_EINVAL;
  if (d.seqlen > 0 && !a.y.data && ((normed_y && a.dy.data) || a.dgate || a.dpost_weight)) return LITE_ATTN_EINVAL;
  bool sums = false;
  for (const float* g : {a.dgate, a.dscale, a.dshift, a.dpost_weight, a.dpre_weight, a.dpre_bias}) {
    if (!good_grad(g)) return LITE_ATTN_EINVAL;
    sums = sums || g;
  }
  if (!sums && !a.dx.data && !a.dy.data) return LITE_ATTN_EINVAL;
  if (sums && (!a.workspace || ((uintptr_t)a.workspace & 15) ||
               a.workspace_bytes < lite_attn_residual_norm_bwd_workspace(&d)))
    return LITE_ATTN_EWORKSPACE;
  auto take = [&](const lite_attn_rows_t& t, int dtype, bool result, Lines* to) {
    *to = lines(t, dtype);
    return !t.data || good(view(t, d.batch, d.seqlen, d.dim, dtype), result);
  };
  if (!take(a.dh, d.dtype, false, &p->dh) || !take(a.dx_out, d.stream_dtype, false, &p->dxo) ||
      !take(a.x_out, d.stream_dtype, false, &p->x) || !take(a.y, d.dtype, false, &p->y) ||
      !take(a.dx, d.stream_dtype, true, &p->dx) || !take(a.dy, d.dtype, true, &p->dy))
    return LITE_ATTN_EINVAL;
  if (sums) {
    p->part = static_cast<float*>(a.workspace);
    p->group_sums = p->part + 3 * (size_t)d.batch * p->groups * s.shares * d.dim;
    p->dgate = a.dgate;
    p->dscale = a.dscale;
    p->dshift = a.dshift;
    p->dpost_w = a.dpost_weight;
    p->dpre_w = a.dpre_weight;
    p->dpre_b = a.dpre_bias;
  }
  return launch_of((int64_t)d.batch * p->groups, s.shares, s.threads, l);
}

}  // namespace la

extern "C" {

size_t lite_attn_rotary_bwd_workspace(const lite_attn_rotary_desc_t* desc) {
  if (la::check_rotary(desc) != LITE_ATTN_OK || desc->norm == LITE_ATTN_NORM_NONE) return 0;
  // (which of the two shapes a call takes depends on its strides)
  return std::max(la::rotary_workspace(*desc, la::rotary_shape(*desc, true, la::kOneByOne)),
                  la::rotary_workspace(*desc, la::rotary_shape(*desc, true, la::kTogether)));
}

size_t lite_attn_residual_norm_bwd_workspace(const lite_attn_residual_desc_t* desc) {
  if (la::check_residual(desc) != LITE_ATTN_OK) return 0;
  const size_t rows = (size_t)desc->batch * la::groups_of(*desc) * (la::residual_shape(*desc, true).shares + 1);
  return la::up16(3 * sizeof(float) * rows * desc->dim);
}

int lite_attn_rotary_freqs(const int32_t axis_pairs[3], double theta, double* host_freqs) {
  if (!axis_pairs || !host_freqs || !(theta > 0.0) || !std::isfinite(theta)) return LITE_ATTN_EINVAL;
  int64_t pairs = 0;
  for (int a = 0; a < 3; ++a) {
    if (axis_pairs[a] < 0 || axis_pairs[a] > 256) return LITE_ATTN_EINVAL;
    pairs += axis_pairs[a];
  }
  int64_t at = 0;
  for (int a = 0; a < 3; ++a) {
    for (int64_t x = 0; x < pairs; ++x) {
      const bool mine = x >= at && x < at + axis_pairs[a];
      host_freqs[a * pairs + x] = mine ? std::pow(theta, -(double)(x - at) / axis_pairs[a]) : 0.0;
    }
    at += axis_pairs[a];
  }
  return LITE_ATTN_OK;
}

}  // extern "C"
