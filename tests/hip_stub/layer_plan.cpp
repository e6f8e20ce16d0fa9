// TEST INFRASTRUCTURE: the host side of the layer operators on random calls, without a device.  What a launch is planned to do is
// walked through here the way the kernels go about it -- workgroup, thread, tile by tile -- and checked against the tensors of
// the call: every entry of every result is written once, none outside of it, nothing is read outside of an input, offsets fit 32
// bits, the sums' places are all different and inside the workspace, and the passes behind read the places that were written.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <set>
#include <vector>

#include "lite_attn_kernels.h"
#include "lite_attn_layer_kernels.h"

#define CHECK(x)                                                                  \
  do {                                                                            \
    if (!(x)) {                                                                   \
      fprintf(stderr, "call %d, line %d: %s\n", call, __LINE__, #x);              \
      exit(1);                                                                    \
    }                                                                             \
  } while (0)

namespace {

std::mt19937 rng(20251206);
int call = 0;
int pick(int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); }
template <class T>
T one_of(std::initializer_list<T> l) {
  return l.begin()[rng() % l.size()];
}

// A tensor's memory begins here; nothing is read.
char* const base = reinterpret_cast<char*>((uintptr_t)1 << 40);

lite_attn_heads_t heads(int batch, int h, int n, int d, int size, int64_t* bytes, bool wide) {
  lite_attn_heads_t t;
  t.data = base;
  const int64_t gap = wide ? (int64_t)1 << 30 : pick(0, 2) * 8;
  if (pick(0, 1)) {  // heads first
    t.stride_n = d + gap;
    t.stride_h = n * t.stride_n;
    t.stride_b = h * t.stride_h;
  } else {
    t.stride_h = d;
    t.stride_n = h * d + gap;
    t.stride_b = n * t.stride_n;
  }
  *bytes = ((batch - 1) * t.stride_b + (h - 1) * t.stride_h + (n - 1) * t.stride_n + d) * size;
  return t;
}

void rotary(bool bwd) {
  lite_attn_rotary_desc_t d = {};
  const bool large = pick(0, 9) == 0;
  d.batch = pick(1, 3);
  d.seqlen = large ? pick(1000, 6000) : pick(1, 60);
  d.heads_q = pick(1, large ? 3 : 20);
  d.heads_k = one_of({0, 1, d.heads_q, std::max(1, d.heads_q / 3)});
  d.head_dim = 2 * (large ? pick(1, 40) : pick(1, 256));
  d.pairs = pick(0, d.head_dim / 2);
  d.halves = pick(0, 1);
  d.dtype = pick(0, 2);
  d.weight_dtype = pick(0, 2);
  d.norm = pick(0, 2);
  d.grid[0] = pick(1, 5), d.grid[1] = pick(1, 9), d.grid[2] = pick(1, 9);
  d.eps = 1e-6f;
  if (la::check_rotary(&d) != LITE_ATTN_OK) return;
  const int size = d.dtype == LITE_ATTN_F32 ? 4 : 2;
  const bool wide = pick(0, 7) == 0, normed = d.norm != LITE_ATTN_NORM_NONE;
  int64_t in_bytes[2], out_bytes[2], g_bytes[2];
  lite_attn_heads_t in[2], out[2], g[2];
  for (int x = 0; x < 2; ++x) {
    const int h = x ? std::max(1, d.heads_k) : d.heads_q;
    in[x] = heads(d.batch, h, d.seqlen, d.head_dim, size, &in_bytes[x], wide);
    out[x] = heads(d.batch, h, d.seqlen, d.head_dim, size, &out_bytes[x], false);
    g[x] = heads(d.batch, h, d.seqlen, d.head_dim, size, &g_bytes[x], false);
  }
  lite_attn_positions_t at = {reinterpret_cast<const double*>(base), nullptr, 0, pick(0, 500)};
  la::RotaryParams p;
  la::LayerLaunch l;
  const size_t space = lite_attn_rotary_bwd_workspace(&d);
  float w;
  int rc;
  if (bwd) {
    lite_attn_rotary_bwd_t a = {in[0], in[1], g[0], g[1], out[0], out[1], nullptr, nullptr, at, normed ? &w : nullptr,
                                normed ? &w : nullptr, base, space};
    rc = la::plan_rotary(d, a, &p, &l);
  } else {
    lite_attn_rotary_fwd_t a = {in[0], in[1], out[0], out[1], nullptr, nullptr, at};
    rc = la::plan_rotary(d, a, &p, &l);
  }
  if (rc == LITE_ATTN_EUNSUPPORTED && wide) return;
  CHECK(rc == LITE_ATTN_OK);
  CHECK(l.threads % 64 == 0 && l.threads <= (l.sums == la::kSumWaves ? la::kMaxTeam : 256));
  const int sides = la::rotary_sides(normed, bwd);
  std::vector<std::vector<char>> seen(2);
  for (int x = 0; x < p.sides; ++x) seen[x].resize((size_t)d.batch * p.side[x].heads * d.seqlen * ((d.head_dim + 7) / 8));
  std::set<const float*> places;
  CHECK(4 * p.lanes * p.tokens <= la::kAngles);
  for (int bi = 0; bi < l.blocks; ++bi) {
    const int per_xcd = l.blocks >> 3, rest = l.blocks & 7, xcd = bi & 7;
    const int place = p.shared_reads ? xcd * per_xcd + std::min(xcd, rest) + (bi >> 3) : bi;
    const int block = sides == 2 ? place : place / p.sides, which = sides == 2 ? 0 : place - block * p.sides;
    const int share = block / p.groups, group = block - share * p.groups;
    const int batch = share / p.shares, n0 = (share - batch * p.shares) * p.tokens, step = p.shares * p.tokens;
    CHECK(batch < d.batch && n0 < d.seqlen);
    for (int s = which; s < (sides == 2 ? p.sides : which + 1); ++s) {
      const la::RotarySide& side = p.side[s];
      if (side.part) {  // what the weights' sums are left in
        const int rows = p.by_row ? p.tokens * side.heads : 1;
        const float* to = side.part + (p.by_row ? (size_t)share * p.tokens * side.heads : (size_t)block) * d.head_dim;
        if (!p.by_row || group == 0) {
          CHECK(places.insert(to).second);
          CHECK((const char*)(to + rows * d.head_dim) <= base + space);
        }
      }
      for (int tid = 0; tid < l.threads; ++tid) {
        const int sub = la::quotient(tid, p.row_lanes, p.per_row), in_row = tid - sub * p.row_lanes;
        const int slot = la::quotient(in_row, p.lanes, p.per_lanes), c = in_row - slot * p.lanes;
        CHECK(sub == tid / p.row_lanes && slot == in_row / p.lanes);
        const int head = group * p.team_heads + slot;
        const int in_head = sub < p.tokens && slot < p.team_heads ? std::min(4, d.head_dim / 2 - 4 * c) : 0;
        if (head >= side.heads || in_head <= 0) continue;
        if (l.sums == la::kSumLanes) CHECK(tid / (1 << p.sum_log) == (tid - (p.by_row ? in_row : c)) / (1 << p.sum_log));
        const int first_of_wave = (tid & ~63) - la::quotient(tid & ~63, p.row_lanes, p.per_row) * p.row_lanes;
        const int wave_slot = p.tokens > 1 ? 0 : la::quotient(first_of_wave, p.lanes, p.per_lanes);
        const int wave_head = group * p.team_heads + wave_slot;
        for (int n = n0; n < d.seqlen; n += step) {
          if (n + sub >= d.seqlen) continue;
          char& once = seen[s][(((size_t)batch * side.heads + head) * d.seqlen + n + sub) * ((d.head_dim + 7) / 8) + c];
          CHECK(!once);
          once = 1;
          auto inside = [&](const char* data, const int64_t* st, int64_t bytes) {
            const int64_t span = (std::min(p.near_heads, side.heads) - 1) * st[1] + (p.tokens - 1) * st[2] + d.head_dim * size;
            const int64_t off = (slot - wave_slot) * st[1] + sub * st[2];
            const int64_t from = data - base + batch * st[0] + n * st[2] + wave_head * st[1] + off;
            return span <= ((int64_t)1 << 32) - 4096 && off >= 0 && off + d.head_dim * size <= span && from >= 0 &&
                   from + d.head_dim * size <= bytes;
          };
          if (!bwd || normed) CHECK(inside(side.x, side.xs, in_bytes[s]));
          if (bwd) CHECK(inside(side.g, side.gs, g_bytes[s]));
          CHECK(inside(side.out, side.os, out_bytes[s]));
        }
      }
    }
  }
  for (int x = 0; x < p.sides; ++x)
    for (char once : seen[x]) CHECK(once);
}

void residual(bool bwd) {
  lite_attn_residual_desc_t d = {};
  d.batch = pick(1, 4);
  d.seqlen = pick(0, 7) == 0 ? pick(1000, 9000) : pick(1, 80);
  d.dim = pick(0, 1) ? pick(1, 600) : pick(600, 8192);
  d.tokens_per_mod = one_of({1, d.seqlen, 2 * d.seqlen, pick(1, d.seqlen), pick(1, d.seqlen)});
  d.dtype = pick(0, 2);
  d.stream_dtype = one_of({d.dtype, (int32_t)LITE_ATTN_F32});
  d.param_dtype = pick(0, 2);
  d.post_norm = one_of({0, 3, 4});
  d.pre_norm = one_of({0, 3, 4});
  d.residual_scale = 1.f;
  CHECK(la::check_residual(&d) == LITE_ATTN_OK);
  const int64_t gap = pick(0, 2) * 8;
  lite_attn_rows_t t = {base, d.seqlen * (d.dim + gap), d.dim + gap}, none = {};
  la::ResidualParams p;
  la::LayerLaunch l;
  const size_t space = lite_attn_residual_norm_bwd_workspace(&d);
  float w;
  if (bwd) {
    lite_attn_residual_bwd_t a = {t, t, t, t, t, t, none, none, nullptr, nullptr, nullptr, &w, &w, &w, &w, &w, &w, base, space};
    CHECK(la::plan_residual(d, a, &p, &l) == LITE_ATTN_OK);
  } else {
    lite_attn_residual_fwd_t a = {t, t, t, t, none, none, none, nullptr, nullptr, nullptr};
    CHECK(la::plan_residual(d, a, &p, &l) == LITE_ATTN_OK);
  }
  const int groups = (d.seqlen + d.tokens_per_mod - 1) / d.tokens_per_mod;
  CHECK(p.groups == groups && l.threads % 64 == 0 && l.threads <= la::kMaxTeam && l.threads * la::kEach >= d.dim);
  CHECK(l.threads * la::kEach < d.dim + 64 * la::kEach);  // (no wave without a column)
  CHECK(l.blocks == d.batch * groups * p.shares);
  std::vector<char> seen((size_t)d.batch * d.seqlen), left((size_t)l.blocks);
  for (int b = 0; b < l.blocks; ++b) {
    const int g = b / p.shares, batch = g / p.groups, group = g - batch * p.groups;
    const int n0 = group * p.per_mod + (b - g * p.shares), end = std::min(p.N, (group + 1) * p.per_mod);
    if (n0 >= end) continue;
    for (int n = n0; n < end; n += p.shares) {
      CHECK(n / d.tokens_per_mod == group);
      char& once = seen[(size_t)batch * d.seqlen + n];
      CHECK(!once);
      once = 1;
    }
    left[b] = 1;
    if (bwd) CHECK((const char*)(p.part + 3 * (size_t)(b + 1) * d.dim) <= (const char*)p.group_sums);
  }
  for (char once : seen) CHECK(once);
  if (!bwd) return;
  CHECK((const char*)(p.group_sums + 3 * (size_t)d.batch * groups * d.dim) <= base + space);
  for (int group = 0; group < d.batch * groups; ++group) {  // the shares that group_sums_kernel reads
    const int g = group % p.groups;
    const int shares = std::min(p.shares, std::min(p.N, (g + 1) * p.per_mod) - g * p.per_mod);
    for (int x = 0; x < p.shares; ++x) CHECK(left[(size_t)group * p.shares + x] == (x < shares));
  }
}

}  // namespace

int main() {
  for (call = 0; call < 1500; ++call) {
    rotary(call & 1);
    residual(call & 1);
  }
  printf("layer plan ok\n");
  return 0;
}
