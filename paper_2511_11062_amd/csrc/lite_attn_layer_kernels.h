// Internal interface between the host side of include/lite_attn_layer.h and its kernels (not installed).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "lite_attn_layer.h"

namespace la {

// Both operators go over rows (a token, or some heads of one) with workgroups whose threads hold kEach entries of the row
// each and that take several rows with the same weights, gate, scale and shift: these, and sums over tokens, stay in
// registers from row to row.  Workgroups that run side by side take neighbouring rows, and all of them move on by the same
// step: what they have under way at any time lies close together in memory (shares of consecutive rows, a window for each
// workgroup, reach 5.0 TB/s where this reaches 5.8, in a copy of 1.5 GB).
constexpr int kEach = 8;
constexpr int kMaxTeam = 1024;
constexpr int kAngles = 1024;  // angles of the tokens that a workgroup keeps at a time, 8 bytes each

// One of q and k.
struct RotarySide {
  const char* x;      // input (backwards: of the forward pass; null if it is not read)
  const char* g;      // backwards: gradient of the result
  char* out;          // result (backwards: gradient of the input)
  int64_t xs[3], gs[3], os[3];  // strides over batch, heads, tokens, bytes
  const void* w;      // weights or null
  float* part;        // backwards: sums for the weights' gradient, [batch * shares][tokens][heads][head_dim] or, of weights
                      //   that the heads share, [batch * shares][groups][head_dim]; or null
  float inv_count;    // 1 / entries that a norm goes over
  int heads;
};

// What a norm's sums go over: no norm; neighbouring lanes, a power of two of them; the lanes of a head, by way of LDS; all waves
// of the workgroup.
enum Sums { kSumNone, kSumLanes, kSumHeads, kSumWaves };
// Of q and k, how many a workgroup takes.
constexpr int rotary_sides(bool normed, bool bwd) { return bwd && normed ? 1 : 2; }

struct RotaryParams {
  RotarySide side[2];
  int sides;             // 2, or 1: there is no k
  const double* freqs;
  const int32_t* positions;
  int64_t positions_stride_b;
  int batch, N;
  int tokens;            // neighbouring tokens that a workgroup takes at a time, a tile
  int shares;            // share x of a batch entry: tiles x, x + shares, x + 2 shares, ...
  int head_dim, pairs;
  int lanes;             // threads of a head
  int team_heads;        // heads that a workgroup takes, of q and of k
  int groups;            // of as many heads
  int near_heads;        // heads that offsets from one place reach: the workgroup's or, if it takes one token, a wave's
  int row_lanes;         // threads of a token: of its heads, under NORM_ROW up to 64 rounded up to a power of two
  int sum_log;           // kSumLanes: sums go over 1 << sum_log neighbouring lanes
  int by_row, halves, weight_dtype;  // by_row: NORM_ROW
  int shared_reads, shared_writes;  // neighbouring tokens share lines of memory, of an input or a result; of a result
  int token_start, area, width, video;  // area = height * width, video = frames * area
  float eps;
  uint32_t per_area, per_width, per_lanes, per_row, per_tokens, per_angles;  // reciprocals for quotient()
};

// Rows of a tensor: the first of the first batch entry, and strides over batch entries and rows, bytes.
struct Lines {
  char* data;
  int64_t stride_b, stride_n;
};

struct ResidualParams {
  Lines x, y, x_out, h;   // backwards: x is x_out as stored
  Lines dh, dxo, dx, dy;
  Lines gate, scale, shift;
  const void *post_w, *pre_w, *pre_b;
  int batch, N, D, per_mod, groups;  // groups of a batch entry
  int shares;                        // share x of a group's rows, the first being n0: n0 + x, n0 + x + shares, ...
  int post, pre, param_dtype;
  float post_eps, pre_eps, alpha, inv_D;
  float* part;                       // backwards: [batch * groups][shares][3][D] sums, or null
  float *dgate, *dscale, *dshift, *dpost_w, *dpre_w, *dpre_b;
  float* group_sums;                 // [batch * groups][3][D]: the groups' parts of the weights' gradients
};

struct LayerLaunch {
  int threads, blocks;
  Sums sums;  // rotary
};

// lite_attn_layer_host.cpp (no HIP calls): checks, and what a call launches
int check_rotary(const lite_attn_rotary_desc_t* d);
int plan_rotary(const lite_attn_rotary_desc_t& d, const lite_attn_rotary_fwd_t& a, RotaryParams* p, LayerLaunch* l);
int plan_rotary(const lite_attn_rotary_desc_t& d, const lite_attn_rotary_bwd_t& a, RotaryParams* p, LayerLaunch* l);
int check_residual(const lite_attn_residual_desc_t* d);
int plan_residual(const lite_attn_residual_desc_t& d, const lite_attn_residual_fwd_t& a, ResidualParams* p, LayerLaunch* l);
int plan_residual(const lite_attn_residual_desc_t& d, const lite_attn_residual_bwd_t& a, ResidualParams* p, LayerLaunch* l);

// lite_attn_layer.hip
hipError_t launch_rotary(const RotaryParams& p, const LayerLaunch& l, int dtype, bool bwd, hipStream_t st);
hipError_t launch_rotary_weights(const RotaryParams& p, float* dq_weight, float* dk_weight, hipStream_t st);
hipError_t launch_residual(const ResidualParams& p, const LayerLaunch& l, int dtype, int stream_dtype, bool bwd,
                           hipStream_t st);
hipError_t launch_residual_sums(const ResidualParams& p, hipStream_t st);

}  // namespace la
