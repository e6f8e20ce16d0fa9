// gfx950 kernels of include/lite_attn_layer.h and its entry points.
//
//   rotary_kernel          : q and k -> normalised, turned, laid out anew; backwards the gradients of that, and sums for the
//                            weights
//   residual_fwd_kernel    : stream + gate * norm(branch) -> stream, and its norm, scaled and shifted
//   residual_bwd_kernel    : the gradients, and per share of rows three sums for gate, scale, shift and the weights
//   sum_rows_kernel, group_sums_kernel, weight_sums_kernel : the shares' sums, in one fixed order
//
// All of them move some bytes for each of a few operations: they are bound by memory, and everything here serves to keep
// enough bytes in flight and to do nothing twice.  A row is read once: its entries stay in the registers of a workgroup, eight
// in a thread, until its statistics are known.  A workgroup takes every so many-th row, asks for its next one before it works on
// this one, and keeps what belongs to its columns -- weights, gate, scale, shift, sums over tokens -- in registers all the while.
// Sums over a row go through DPP inside a wave and once through LDS between waves.  Bytes that have to move, us and TB/s, where a
// sum of two large tensors reaches 6.2 TB/s:
//   rotary     40 heads of 128, 75600 tokens, norm over the token             3097 MB  652  4.8
//              12 heads, 32760 tokens                                          402 MB   82  4.9
//              the same backwards                                              604 MB  117  5.2
//   residual   75600 x 5120, both norms, a row of modulation for 3600 tokens  3097 MB  599  5.2
//              32760 x 1536, stream in 32 bits                                 604 MB  104  5.8
//              the same backwards                                              906 MB  157  5.8
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "lite_attn_kernels.h"
#include "lite_attn_layer_kernels.h"

namespace la {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Element types: two of them as they lie in a word of memory (F32: one), and the word of two values, each rounded once.
struct Bf16 {
  typedef __bf16 type;
  static __device__ __forceinline__ f32x2 widen(uint32_t w) {
    return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  }
  static __device__ __forceinline__ uint32_t narrow(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
  }
};
struct F16 {
  typedef _Float16 type;
  static __device__ __forceinline__ f32x2 widen(uint32_t w) {
    return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
  }
  static __device__ __forceinline__ uint32_t narrow(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
  }
};
struct F32 {
  typedef float type;
};

// Rows of a tensor, one after the other, read and written through a buffer descriptor: what lies behind the row, or in no row at
// all, reads as 0 and is not written.  So loads and stores stand in no branch, the compiler counts those in flight, and a wait
// for a row that was asked for ahead does not wait for the stores behind it.  Offsets need the alignment of an element only.
typedef __amdgpu_buffer_rsrc_t Buffer;
constexpr int kBufferFlags = 0x00020000;
// Cache policy of rows (bit 1, non-temporal): each is read or written once and makes room at once.  us without -> with,
// forwards 32760 x 1536 (stream in 32 bits) 111 -> 104, backwards 164 -> 158, 75600 x 5120 (bf16) 584 -> 542, rotary of 12
// heads 83.5 -> 82, backwards 125 -> 117, of 40 heads 635 -> 655.
constexpr int kStreamed = 2;
struct Walk {
  char* at;
  int64_t stride;
  int bytes;  // of a row
  __device__ __forceinline__ Buffer row() const { return __builtin_amdgcn_make_buffer_rsrc(at, 0, bytes, kBufferFlags); }
  __device__ __forceinline__ Buffer row_if(bool there) const {
    return __builtin_amdgcn_make_buffer_rsrc(at, 0, there ? bytes : 0, kBufferFlags);
  }
  __device__ __forceinline__ void step() { at += stride; }
};

// Stores that are dropped.  Before a loop that asks for a row ahead, as many as a row has behind that: the compiler counts what
// is in flight at the loop's head by the way with the least, and would otherwise wait for a row's stores where it waits for the
// next row.
template <int kCount>
__device__ __forceinline__ void no_stores(const Walk& to) {
#pragma unroll
  for (int x = 0; x < kCount; ++x) __builtin_amdgcn_raw_buffer_store_b32(0u, to.row_if(false), 0, 0, 0);
}

// Eight entries of a row as they lie in memory, in two runs of four.
template <class Kind>
struct Piece {
  typedef typename Kind::type T;
  static constexpr bool kNarrow = sizeof(T) == 2;
  static constexpr int kSize = sizeof(T);
  uint32_t w[kNarrow ? 4 : 8];

  __device__ __forceinline__ void load_run(int run, Buffer from, int offset) {
    if constexpr (kNarrow) {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(from, offset, 0, kStreamed);
      w[2 * run] = v[0];
      w[2 * run + 1] = v[1];
    } else {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(from, offset, 0, kStreamed);
#pragma unroll
      for (int x = 0; x < 4; ++x) w[4 * run + x] = v[x];
    }
  }
  __device__ __forceinline__ void load(Buffer from, int offset) {
    if constexpr (kNarrow) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(from, offset, 0, kStreamed);
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = v[x];
    } else {
      load_run(0, from, offset);
      load_run(1, from, offset + 16);
    }
  }
  // Entries e and e + 1, each from a place of its own.
  __device__ __forceinline__ void load_two(int e, Buffer from, int offset0, int offset1) {
    if constexpr (kNarrow) {
      const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(from, offset0, 0, kStreamed);
      const uint32_t hi = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(from, offset1, 0, kStreamed);
      w[e / 2] = lo | hi << 16;
    } else {
      w[e] = __builtin_amdgcn_raw_buffer_load_b32(from, offset0, 0, kStreamed);
      w[e + 1] = __builtin_amdgcn_raw_buffer_load_b32(from, offset1, 0, kStreamed);
    }
  }
  __device__ __forceinline__ void unpack(float* x) const {
#pragma unroll
    for (int e = 0; e < kEach; e += 2) {
      f32x2 v;
      if constexpr (kNarrow)
        v = Kind::widen(w[e / 2]);
      else
        v = f32x2{__uint_as_float(w[e]), __uint_as_float(w[e + 1])};
      x[e] = v[0];
      x[e + 1] = v[1];
    }
  }
  __device__ __forceinline__ void pack(const float* x) {
#pragma unroll
    for (int e = 0; e < kEach; e += 2) {
      if constexpr (kNarrow) {
        w[e / 2] = Kind::narrow(x[e], x[e + 1]);
      } else {
        w[e] = __float_as_uint(x[e]);
        w[e + 1] = __float_as_uint(x[e + 1]);
      }
    }
  }
  template <int kPolicy = kStreamed>
  __device__ __forceinline__ void store_run(int run, Buffer to, int offset) const {
    if constexpr (kNarrow)
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{w[2 * run], w[2 * run + 1]}, to, offset, 0, kPolicy);
    else
      __builtin_amdgcn_raw_buffer_store_b128(u32x4{w[4 * run], w[4 * run + 1], w[4 * run + 2], w[4 * run + 3]}, to, offset, 0,
                                             kPolicy);
  }
  template <int kPolicy = kStreamed>
  __device__ __forceinline__ void store(Buffer to, int offset) const {
    if constexpr (kNarrow) {
      __builtin_amdgcn_raw_buffer_store_b128(u32x4{w[0], w[1], w[2], w[3]}, to, offset, 0, kPolicy);
    } else {
      store_run<kPolicy>(0, to, offset);
      store_run<kPolicy>(1, to, offset + 16);
    }
  }
  template <int kPolicy = kStreamed>
  __device__ __forceinline__ void store_two(int e, Buffer to, int offset0, int offset1) const {
    if constexpr (kNarrow) {
      __builtin_amdgcn_raw_buffer_store_b16((uint16_t)w[e / 2], to, offset0, 0, kPolicy);
      __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(w[e / 2] >> 16), to, offset1, 0, kPolicy);
    } else {
      __builtin_amdgcn_raw_buffer_store_b32(w[e], to, offset0, 0, kPolicy);
      __builtin_amdgcn_raw_buffer_store_b32(w[e + 1], to, offset1, 0, kPolicy);
    }
  }
};

__device__ __forceinline__ float load_param(const void* p, int dtype, int64_t at) {
  if (dtype == LITE_ATTN_F32) return static_cast<const float*>(p)[at];
  if (dtype == LITE_ATTN_BF16) return (float)static_cast<const __bf16*>(p)[at];
  return (float)static_cast<const _Float16*>(p)[at];
}

// ---- sums over a team --------------------------------------------------------------------------------------------------

template <int kCtrl>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), kCtrl, 0xf, 0xf, true));
}
__device__ __forceinline__ float add_row_pairs(float x) {  // rows of 16 lanes, 0 with 1 and 2 with 3
  const u32x2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float add_halves(float x) {  // lanes 0..31 with 32..63
  const u32x2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
__device__ __forceinline__ float sum16(float x) {
  return add_dpp<kMirror>(add_dpp<kHalfMirror>(add_dpp<kXor2>(add_dpp<kXor1>(x))));
}
__device__ __forceinline__ float sum64(float x) { return add_halves(add_row_pairs(sum16(x))); }
// Sum over 1 << log neighbouring lanes, in all of them: six steps, those that are too many adding 0.
template <int kStep>
__device__ __forceinline__ float step_of(float x) {
  if constexpr (kStep == 4) {
    const u32x2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 16 ? s[0] : s[1]);
  } else if constexpr (kStep == 5) {
    const u32x2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 32 ? s[0] : s[1]);
  } else {
    constexpr int kCtrl = kStep == 0 ? kXor1 : kStep == 1 ? kXor2 : kStep == 2 ? kHalfMirror : kMirror;
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), kCtrl, 0xf, 0xf, true));
  }
}
template <int kStep = 0>
__device__ __forceinline__ float sum_lanes(float x, int log) {
  if constexpr (kStep < 6) {
    const uint32_t on = log > kStep ? 0xffffffffu : 0u;
    return sum_lanes<kStep + 1>(x + __uint_as_float(__float_as_uint(step_of<kStep>(x)) & on), log);
  } else {
    return x;
  }
}

// A barrier that orders LDS alone: loads and stores of global memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What the waves of a workgroup tell each other: kCount pairs of values each.  The two halves of a room serve in turn: a wave that
// is one exchange ahead cannot overwrite what another still reads, as there is a barrier between.
template <int kCount>
struct WaveRoom {
  f32x2 v[2][kCount][kMaxTeam / 64];
  // This wave's values -> those of wave threadIdx.x % 16 (0 if there is none).
  template <int kUsed>
  __device__ __forceinline__ void exchange(int& turn, f32x2 (&x)[kUsed]) {
    static_assert(kUsed <= kCount, "room for them");
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < kUsed; ++i) v[turn][i][threadIdx.x >> 6] = x[i];
    }
    lds_barrier();
    const int w = threadIdx.x & 15;
    const bool there = w < (int)(blockDim.x >> 6);
#pragma unroll
    for (int i = 0; i < kUsed; ++i) {
      x[i] = v[turn][i][w];
      if (!there) x[i] = f32x2{0.f, 0.f};
    }
    turn ^= 1;
  }
};

// ---- rotary positions --------------------------------------------------------------------------------------------------

// Brings a kernel's arguments into the scalar cache, all lines of 64 bytes at once: they come from host memory, and left to the
// places of their first use a workgroup would wait for one line after the other.
template <int kBytes>
__device__ __forceinline__ void touch_arguments() {
  typedef const __attribute__((address_space(4))) uint32_t* Words;
  const Words a = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  uint32_t x = 0;
#pragma unroll
  for (int line = 0; line < (kBytes + 63) / 64; ++line) x |= a[min(16 * line, kBytes / 4 - 1)];
  asm volatile("" ::"s"(x));
}

// x, of which the compiler does not know that it is the same for each row: what follows from it is made where it is needed, and
// not kept in a register each for all rows.
__device__ __forceinline__ int afresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A kernel's arguments where they lie, to be read there again: what is needed once for many rows takes no scalar registers in
// between.
typedef const __attribute__((address_space(4))) RotaryParams* RotaryArgs;
__device__ __forceinline__ RotaryArgs rotary_args() {
  RotaryArgs a = (RotaryArgs)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return a;
}

// Where a token stands.
struct Position {
  int at[3];
};
__device__ __forceinline__ Position position_of(RotaryArgs p, int batch, int n) {
  if (p->positions) {
    const int32_t* const at = p->positions + batch * p->positions_stride_b + n;
    return {{at[0], at[(int64_t)p->N], at[2 * (int64_t)p->N]}};
  }
  int t = p->token_start + n;
  if (t >= p->video) t = 0;
  const int f = quotient(t, p->area, p->per_area), in = t - f * p->area, y = quotient(in, p->width, p->per_width);
  return {{f, y, in - y * p->width}};
}

// How fast a pair turns, and its cos and sin at a position.  In 64 bits until whole turns are off: in 32 an angle of 10^5
// radians would be off by 6e-3.
struct Speed {
  double f[3];
};
__device__ __forceinline__ Speed speed_of(RotaryArgs p, int pair) {
  const int pairs = p->pairs;
  if (pair >= pairs) return {{0.0, 0.0, 0.0}};
  return {{p->freqs[pair], p->freqs[pairs + pair], p->freqs[2 * pairs + pair]}};
}
__device__ __forceinline__ f32x2 angle_of(const Speed& v, const Position& at) {
  double turns = (double)at.at[0] * v.f[0];
  turns = __builtin_fma((double)at.at[1], v.f[1], turns);
  turns = __builtin_fma((double)at.at[2], v.f[2], turns);
  turns *= 0.15915494309189533577;  // 1 / (2 pi)
  turns -= __builtin_rint(turns);
  float s, c;
  sincospif(2.f * (float)turns, &s, &c);
  return f32x2{c, s};
}

// The angles of `tiles` tiles of tokens, the first of them at token n, `step` tokens from one to the next: 4 * lanes for each
// token.  If those are whole waves, a wave takes a token, whose position it finds by scalar instructions, and a thread keeps its
// pair (`mine`: how fast pair threadIdx.x % 64 turns).
__device__ __forceinline__ void make_angles(const Speed& mine, int batch, int n, int step, int tiles, f32x2* angles) {
  const RotaryArgs p = rotary_args();
  const int each = 4 * p->lanes, tokens = tiles * p->tokens;
  auto token = [&](int x) {  // (of the last tile some may be none)
    const int tile = quotient(x, p->tokens, p->per_tokens);
    return min(p->N - 1, n + tile * step + (x - tile * p->tokens));
  };
  if (each % 64 == 0) {
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int first = 0; first < each; first += 64) {
      const Speed v = first == 0 ? mine : speed_of(p, first + lane);
      for (int x = wave; x < tokens; x += waves)
        angles[x * each + first + lane] = angle_of(v, position_of(p, batch, token(x)));
    }
  } else {
    for (int x = threadIdx.x; x < tokens * each; x += blockDim.x) {
      const int t = quotient(x, each, p->per_angles);
      angles[x] = angle_of(speed_of(p, x - t * each), position_of(p, batch, token(t)));
    }
  }
}

// A workgroup: some heads (under NORM_ROW all) of q and the same heads of k, whose angles are the same, for a share of the
// tokens, one or some at a time.  A row is a token's heads of q or of k, one after the other.  (Backwards through a norm,
// where weights and the sums for their gradient would need 32 registers, a workgroup takes q or k.)  A thread holds four
// pairs of a head, a[4] and b[4]. WHOLE: they are eight entries in a row or, of turned halves, four and four; otherwise (a
// head's ragged end, four pairs across the end of the turned halves) every entry is fetched by itself.
template <class Kind, bool HALVES, bool WHOLE, Sums SUMS, bool BWD>
__global__ __launch_bounds__(SUMS == kSumWaves ? kMaxTeam : 256) void rotary_kernel(const RotaryParams p) {
  constexpr int kSize = Piece<Kind>::kSize;
  constexpr bool kNormed = SUMS != kSumNone;
  constexpr int kSides = rotary_sides(kNormed, BWD);
  touch_arguments<sizeof(RotaryParams)>();
  __shared__ f32x2 angles[kAngles];
  __shared__ WaveRoom<1> room;
  __shared__ f32x2 lane_sums[2][SUMS == kSumHeads ? 256 + 64 : 1];  // (threads of no head read on behind 256)
  const int tid = threadIdx.x;
  // Workgroups go to the XCDs in turn.  Where neighbouring tokens share lines, an XCD takes neighbouring shares, and its cache
  // keeps a result's line until the others have written their parts of it.
  const int per_xcd = (int)gridDim.x >> 3, rest = (int)gridDim.x & 7, xcd = (int)blockIdx.x & 7;
  const int place = p.shared_reads ? xcd * per_xcd + min(xcd, rest) + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
  const int block = kSides == 2 ? place : place / p.sides;
  const int which = kSides == 2 ? 0 : place - block * p.sides;  // of q and k
  const RotarySide* const sides = p.side + which;
  const int share = block / p.groups, group = block - share * p.groups;
  const int batch = share / p.shares, n0 = (share - batch * p.shares) * p.tokens, step = p.shares * p.tokens;

  const int sub = quotient(tid, p.row_lanes, p.per_row), in_row = tid - sub * p.row_lanes;  // token of the tile
  const int slot = quotient(in_row, p.lanes, p.per_lanes), c = in_row - slot * p.lanes;
  const int head = group * p.team_heads + slot;
  // pairs of the head from this thread's first on
  const int in_head = sub < p.tokens && slot < p.team_heads ? min(4, p.head_dim / 2 - 4 * c) : 0;
  auto valid = [&](int side, int e) { return head < sides[side].heads && (WHOLE ? in_head > 0 : e < in_head); };
  // places in the head of a[e] and b[e]
  const int P = p.pairs;
  auto place_a = [&](int e) {
    const int i = 4 * c + e;
    return HALVES && i < P ? i : HALVES ? 2 * P + 2 * (i - P) : 2 * i;
  };
  auto place_b = [&](int e) { return HALVES && 4 * c + e < P ? 4 * c + e + P : place_a(e) + 1; };
  const bool apart = HALVES && 4 * c < P;
  const int first = place_a(0), second = apart ? first + P : first + 4;

  // A wave's rows start at its first head (at the workgroup's, if that takes some tokens); other heads are `stride_h` and other
  // tokens `stride_n` apart.  Entries that are not there lie behind all.
  const int wave_slot = p.tokens > 1 ? 0 : __builtin_amdgcn_readfirstlane(slot);
  const int wave_head = group * p.team_heads + wave_slot;
  struct Tensor {
    Walk walk;
    int first, second;
  };
  auto tensor = [&](int side, const char* data, const int64_t* s) {
    Tensor t;
    const int heads = sides[side].heads;
    const int64_t span = heads == 0 ? 0 : (min(p.near_heads, heads) - 1) * s[1] + (p.tokens - 1) * s[2] + p.head_dim * kSize;
    t.walk = Walk{const_cast<char*>(data) + batch * s[0] + n0 * s[2] + wave_head * s[1], step * s[2], (int)span};
    const int64_t at = (slot - wave_slot) * s[1] + sub * s[2];
    t.first = valid(side, 0) ? (int)(at + first * kSize) : (int)span;
    t.second = valid(side, 0) ? (int)(at + second * kSize) : (int)span;
    return t;
  };
  auto fetch = [&](int side, Tensor& t, bool there, Piece<Kind>& to) {
    const Buffer from = t.walk.row();
    t.walk.step();
    if constexpr (WHOLE && HALVES) {
      to.load_run(0, from, there ? t.first : t.walk.bytes);
      to.load_run(1, from, there ? t.second : t.walk.bytes);
    } else if constexpr (WHOLE) {
      to.load(from, there ? t.first : t.walk.bytes);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = afresh(t.first);
        const int a = there && valid(side, e) ? at + (place_a(e) - first) * kSize : t.walk.bytes;
        const int b = there && valid(side, e) ? at + (place_b(e) - first) * kSize : t.walk.bytes;
        to.load_two(2 * e, from, a, b);
      }
    }
  };
  auto unpack = [&](const auto& from, float* a, float* b) {
    float x[kEach];
    from.unpack(x);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = WHOLE && HALVES && apart ? x[e] : x[2 * e];
      b[e] = WHOLE && HALVES && apart ? x[4 + e] : x[2 * e + 1];
    }
  };
  auto store = [&](int side, Tensor& t, bool there, const float* ra, const float* rb) {
    const Buffer to = t.walk.row();
    t.walk.step();
    float x[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      x[e] = e & 1 ? rb[e / 2] : ra[e / 2];
      if (WHOLE && HALVES && apart) x[e] = e < 4 ? ra[e & 3] : rb[e & 3];
    }
    Piece<Kind> out;
    out.pack(x);
    auto put = [&](auto policy) {
      constexpr int kPolicy = decltype(policy)::value;
      if constexpr (WHOLE && HALVES) {
        out.template store_run<kPolicy>(0, to, there ? t.first : t.walk.bytes);
        out.template store_run<kPolicy>(1, to, there ? t.second : t.walk.bytes);
      } else if constexpr (WHOLE) {
        out.template store<kPolicy>(to, there ? t.first : t.walk.bytes);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = afresh(t.first);
          const int a = there && valid(side, e) ? at + (place_a(e) - first) * kSize : t.walk.bytes;
          const int b = there && valid(side, e) ? at + (place_b(e) - first) * kSize : t.walk.bytes;
          out.template store_two<kPolicy>(2 * e, to, a, b);
        }
      }
    };
    if (p.shared_writes)
      put(std::integral_constant<int, 0>{});
    else
      put(std::integral_constant<int, kStreamed>{});
  };

  Tensor in_x[kSides], in_g[kSides], out[kSides];
#pragma unroll
  for (int side = 0; side < kSides; ++side) {
    const RotarySide& s = sides[side];
    if constexpr (!BWD || kNormed) in_x[side] = tensor(side, s.x, s.xs);
    if constexpr (BWD) in_g[side] = tensor(side, s.g, s.gs);
    out[side] = tensor(side, s.out, s.os);
  }
  Piece<Kind> next_x, next_g;
  auto fetch_next = [&](int side, bool there) {
    if constexpr (!BWD || kNormed) fetch(side, in_x[side], there, next_x);
    if constexpr (BWD) fetch(side, in_g[side], there, next_g);
  };
  fetch_next(0, n0 + sub < p.N);
  const Speed mine = speed_of(rotary_args(), tid & 63);      // (asked for before anything is waited for)
  float wa[kSides][4], wb[kSides][4], da[kSides][4], db[kSides][4];  // weights and, backwards, the sums for their gradient
  if constexpr (kNormed) {
    auto load_weights = [&](auto kind) {
      typedef Piece<decltype(kind)> Weights;
      Weights v[kSides];
#pragma unroll
      for (int side = 0; side < kSides; ++side) {
        const int heads = p.by_row ? sides[side].heads : 1;
        const int bytes = sides[side].w ? heads * p.head_dim * Weights::kSize : 0;
        const Buffer from = Walk{(char*)sides[side].w, 0, bytes}.row();
        const int row = p.by_row ? head * p.head_dim : 0;
#pragma unroll
        for (int e = 0; e < kEach && !WHOLE; e += 2)
          v[side].load_two(e, from, valid(side, e / 2) ? (row + place_a(e / 2)) * Weights::kSize : bytes,
                           valid(side, e / 2) ? (row + place_b(e / 2)) * Weights::kSize : bytes);
        if constexpr (WHOLE) {
          v[side].load_run(0, from, valid(side, 0) ? (row + first) * Weights::kSize : bytes);
          v[side].load_run(1, from, valid(side, 0) ? (row + second) * Weights::kSize : bytes);
        }
      }
#pragma unroll
      for (int side = 0; side < kSides; ++side) {
        unpack(v[side], wa[side], wb[side]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!sides[side].w) wa[side][e] = wb[side][e] = 1.f;
          da[side][e] = db[side][e] = 0.f;
        }
      }
    };
    if (p.weight_dtype == LITE_ATTN_F32)
      load_weights(F32());
    else if (p.weight_dtype == LITE_ATTN_BF16)
      load_weights(Bf16());
    else
      load_weights(F16());
  }
  int turn = 0;
  float ca[4], sa[4];
  // Sums over what the norm goes over (kSumHeads: each lane of a head adds up all of them from LDS).
  auto row_sum = [&](f32x2 x) {
    if constexpr (SUMS == kSumLanes) {
      x[0] = sum_lanes(x[0], p.sum_log);
      if constexpr (BWD) x[1] = sum_lanes(x[1], p.sum_log);
      return x;
    } else if constexpr (SUMS == kSumWaves) {
      x[0] = sum64(x[0]);
      if constexpr (BWD) x[1] = sum64(x[1]);
      f32x2 all[1] = {x};
      room.exchange(turn, all);
      x[0] = sum16(all[0][0]);
      if constexpr (BWD) x[1] = sum16(all[0][1]);
      return x;
    } else {
      lane_sums[turn][tid] = x;
      lds_barrier();
      const f32x2* const mine = &lane_sums[turn][tid - c];
      x = mine[0];
      for (int l = 1; l < p.lanes; ++l) x += mine[l];
      turn ^= 1;
      return x;
    }
  };
  // Entries that are not turned stay what they are: a turn by 0 would make NaN of an entry beside an infinite one.
  auto not_turned = [&](const float* xa, const float* xb, float* ra, float* rb) {
    if (2 * P == p.head_dim) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool turned = 4 * afresh(c) + e < P;
      ra[e] = turned ? ra[e] : xa[e];
      rb[e] = turned ? rb[e] : xb[e];
    }
  };
  // A row; the next one is of `next_side`.
  auto do_row = [&](auto index, bool here, int next_side, bool there) {
    constexpr int side = decltype(index)::value;
    const Piece<Kind> x = next_x, g = next_g;
    if (kSides == 2 && next_side)
      fetch_next(kSides - 1, there);
    else
      fetch_next(0, there);
    const float inv_count = sides[side].inv_count;
    float xa[4], xb[4];
    if constexpr (!BWD) {
      unpack(x, xa, xb);
      if constexpr (kNormed) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sq += xa[e] * xa[e] + xb[e] * xb[e];  // (0 where there is no entry)
        sq = row_sum(f32x2{sq, 0.f})[0];
        const float rstd = rsqrtf(sq * inv_count + p.eps);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xa[e] *= rstd * wa[side][e];
          xb[e] *= rstd * wb[side][e];
        }
      }
      float ra[4], rb[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ra[e] = xa[e] * ca[e] - xb[e] * sa[e];
        rb[e] = xa[e] * sa[e] + xb[e] * ca[e];
      }
      not_turned(xa, xb, ra, rb);
      store(side, out[side], here, ra, rb);
    } else {
      float ga[4], gb[4], za[4], zb[4];
      unpack(g, ga, gb);
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // the turn back
        za[e] = ga[e] * ca[e] + gb[e] * sa[e];
        zb[e] = gb[e] * ca[e] - ga[e] * sa[e];
      }
      not_turned(ga, gb, za, zb);
      if constexpr (kNormed) {
        unpack(x, xa, xb);
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sq += xa[e] * xa[e] + xb[e] * xb[e];
          dot += za[e] * wa[side][e] * xa[e] + zb[e] * wb[side][e] * xb[e];
        }
        const f32x2 all = row_sum(f32x2{sq, dot});
        sq = all[0];
        dot = all[1];
        // n = x rstd; dx = rstd (dn - n mean(dn n)), dn = dz w
        const float rstd = rsqrtf(sq * inv_count + p.eps);
        const float pull = rstd * rstd * (dot * inv_count);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          da[side][e] += za[e] * (xa[e] * rstd);
          db[side][e] += zb[e] * (xb[e] * rstd);
          za[e] = rstd * (za[e] * wa[side][e] - xa[e] * pull);
          zb[e] = rstd * (zb[e] * wb[side][e] - xb[e] * pull);
        }
      }
      store(side, out[side], here, za, zb);
    }
  };

  const int each = 4 * p.lanes * p.tokens;  // angles of a tile, with those of entries that are not turned
  const int some = kAngles / each;          // tiles whose angles are made at a time
  const bool both = kSides == 2 && p.sides == 2;
  int made = 0, at = 0;  // tiles left of those, and where this thread's angles of this one start
  no_stores<!WHOLE ? 8 : HALVES || kSize == 4 ? 2 : 1>(out[0].walk);
  for (int n = n0; n < p.N; n += step) {
    if (made == 0) {
      if (n != n0) lds_barrier();
      made = min(some, (p.N - 1 - n) / step + 1);
      make_angles(mine, batch, n, step, made, angles);
      at = 4 * (min(sub, p.tokens - 1) * p.lanes + c);
      lds_barrier();
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x2 cs = angles[at + e];
      ca[e] = cs[0];
      sa[e] = cs[1];
    }
    at += each;
    --made;
    const bool here = n + sub < p.N, more = n + step + sub < p.N;
    do_row(std::integral_constant<int, 0>{}, here, both, both ? here : more);
    if (both) do_row(std::integral_constant<int, kSides - 1>{}, here, 0, more);
  }

  if constexpr (BWD && kNormed) {
#pragma unroll
    for (int side = 0; side < kSides; ++side) {
      const RotaryArgs args = rotary_args();
      const auto* const s = args->side + (which + side);
      if (!s->part) continue;
      if (args->by_row) {
        float* to = s->part + (((size_t)share * args->tokens + sub) * s->heads + head) * args->head_dim;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!valid(side, e)) continue;
          to[place_a(e)] = da[side][e];
          to[place_b(e)] = db[side][e];
        }
      } else if constexpr (SUMS != kSumWaves) {  // weights that heads share: the tile's tokens and their heads summed in order
        __shared__ float sums[256 * kEach];
        lds_barrier();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sums[tid * kEach + 2 * e] = valid(side, e) ? da[side][e] : 0.f;
          sums[tid * kEach + 2 * e + 1] = valid(side, e) ? db[side][e] : 0.f;
        }
        lds_barrier();
        float* to = s->part + (size_t)block * args->head_dim;
        if (tid < args->lanes) {
          const int rows = args->tokens * args->team_heads;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (e >= in_head) continue;
            float ta = 0.f, tb = 0.f;
            for (int h = 0; h < rows; ++h) {
              ta += sums[(h * args->lanes + c) * kEach + 2 * e];
              tb += sums[(h * args->lanes + c) * kEach + 2 * e + 1];
            }
            to[place_a(e)] = ta;
            to[place_b(e)] = tb;
          }
        }
      }
    }
  }
}

// Part w of n things cut into `parts`: from part_start(w) to part_start(w + 1).
__device__ __forceinline__ int part_start(int n, int parts, int w) { return (int)((int64_t)n * w / parts); }

// out[column] = the sum over `rows` rows of part[row][columns]: a workgroup takes 64 columns, its waves an equal share of the
// rows each.
struct RowSums {
  const float* part[2];
  float* out[2];
  int rows[2], columns[2], blocks0;
};
__global__ __launch_bounds__(1024) void sum_rows_kernel(const RowSums p) {
  __shared__ float sums[16][64];
  const int which = (int)blockIdx.x >= p.blocks0, block = which ? (int)blockIdx.x - p.blocks0 : (int)blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int column = block * 64 + lane, columns = p.columns[which], rows = p.rows[which];
  const int r1 = part_start(rows, 16, wave + 1);
  float sum = 0.f;
  if (column < columns) {
    const float* from = p.part[which] + column;
#pragma unroll 8
    for (int r = part_start(rows, 16, wave); r < r1; ++r) sum += from[(size_t)r * columns];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && column < columns) {
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    p.out[which][column] = sum;
  }
}

// ---- residual stream ---------------------------------------------------------------------------------------------------

// The columns of a row that a thread holds: kEach in a row; four and four, where 32-bit entries are among them, so that the lanes
// of an access of 16 bytes each lie side by side; one of each `team` in rows of fewer than eight.  Rows that are not whole pieces
// (TAIL): the last piece is moved back until it ends with the row.  What it has in common with the one before it is read and
// written by both, the same values, and counts in the other's sums only.  What lies behind the row reads as 0 and is not written.
enum Spread { kEights, kFours, kEightsTail, kFoursTail, kOnes };
constexpr bool has_tail(Spread s) { return s == kEightsTail || s == kFoursTail; }
constexpr int piece_of(Spread s) { return s == kOnes ? 1 : s == kFours || s == kFoursTail ? 4 : 8; }
template <Spread S>
struct Columns {
  int thread, team, D;
  // TAIL, which entries count in this thread's sums: all bits of them, or none (a mask over lanes for each would not fit the
  // scalar registers, and a factor of 0 would make NaN of an infinity that counts elsewhere); of pieces of four, where vector
  // registers are short too, the first of each piece that counts
  uint32_t keep[S == kEightsTail ? kEach : 1];
  int from[2];
  __device__ __forceinline__ Columns(int thread_, int team_, int D_) : thread(thread_), team(team_), D(D_) {
    if constexpr (S == kEightsTail) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        keep[e] = own(e) < D && at(e) >= own(e) ? 0xffffffffu : 0u;
        asm volatile("" : "+v"(keep[e]));  // (or the compiler makes masks over lanes of them)
      }
    } else if constexpr (S == kFoursTail) {
#pragma unroll
      for (int run = 0; run < 2; ++run) from[run] = own(4 * run) < D ? own(4 * run) - start(4 * run) : 4;
    }
  }
  // where the piece of entry e starts: its own place, and the one it is moved to
  __device__ __forceinline__ int own(int e) const { return (e / piece_of(S) * team + thread) * piece_of(S); }
  __device__ __forceinline__ int start(int e) const {
    return has_tail(S) && own(e) < D ? min(own(e), D - piece_of(S)) : own(e);
  }
  __device__ __forceinline__ int at(int e) const { return start(e) + e % piece_of(S); }
  // x as entry e's part of a sum
  __device__ __forceinline__ float part(int e, float x) const {
    if constexpr (S == kEightsTail)
      return __uint_as_float(__float_as_uint(x) & keep[e]);
    else if constexpr (S == kFoursTail)
      return afresh(from[e / 4]) <= e % 4 ? x : 0.f;
    else
      return own(e) < D ? x : 0.f;
  }
};
template <class Kind, Spread S>
constexpr int kRowAccesses = S == kOnes ? kEach : piece_of(S) == 4 ? 2 : Piece<Kind>::kSize / 2;  // loads or stores of a row
template <Spread S, class Kind>
__device__ __forceinline__ void load_row(Buffer from, const Columns<S>& col, Piece<Kind>& to) {
  if constexpr (S == kOnes) {
#pragma unroll
    for (int e = 0; e < kEach; e += 2) to.load_two(e, from, col.at(e) * to.kSize, col.at(e + 1) * to.kSize);
  } else if constexpr (piece_of(S) == 4) {
    to.load_run(0, from, col.at(0) * to.kSize);
    to.load_run(1, from, col.at(4) * to.kSize);
  } else {
    to.load(from, col.at(0) * to.kSize);
  }
}
template <class Kind, Spread S>
__device__ __forceinline__ void store_row(Buffer to, const Columns<S>& col, const float* x) {
  Piece<Kind> out;
  out.pack(x);
  if constexpr (S == kOnes) {
#pragma unroll
    for (int e = 0; e < kEach; e += 2) out.store_two(e, to, col.at(e) * out.kSize, col.at(e + 1) * out.kSize);
  } else if constexpr (piece_of(S) == 4) {
    out.store_run(0, to, col.at(0) * out.kSize);
    out.store_run(1, to, col.at(4) * out.kSize);
  } else {
    out.store(to, col.at(0) * out.kSize);
  }
}
template <class Kind, Spread S>
__device__ __forceinline__ void load_vector(const char* p, const Columns<S>& col, float* to) {
  Piece<Kind> v;
  load_row(Walk{const_cast<char*>(p), 0, col.D * v.kSize}.row(), col, v);
  v.unpack(to);
}
template <Spread S>
__device__ __forceinline__ void load_params(const void* p, int dtype, const Columns<S>& col, float* to, float missing) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) to[e] = missing;
  } else if (dtype == LITE_ATTN_F32) {
    load_vector<F32>(static_cast<const char*>(p), col, to);
  } else if (dtype == LITE_ATTN_BF16) {
    load_vector<Bf16>(static_cast<const char*>(p), col, to);
  } else {
    load_vector<F16>(static_cast<const char*>(p), col, to);
  }
}
// A row of modulation.
template <Spread S>
__device__ __forceinline__ void load_mod(const Lines& l, int dtype, int b, int g, const Columns<S>& col, float* to,
                                         float missing) {
  load_params(l.data ? l.data + b * l.stride_b + g * l.stride_n : nullptr, dtype, col, to, missing);
}

// A row's team, the waves of the workgroup.
struct Team {
  bool waves;  // more than one
  int turn;
  WaveRoom<3>* room;
  template <int kUsed>
  __device__ __forceinline__ void exchange(f32x2 (&x)[kUsed]) {
    if (waves) room->exchange(turn, x);
  }
  // A row may be worked on in place, and two waves may hold the same entries of it (TAIL): all of them are asked for before the
  // waves meet in the row, and stored after that.  Where no norm makes them exchange anything, they meet here.
  template <Spread S>
  __device__ __forceinline__ void meet(bool exchanged) const {
    if (has_tail(S) && waves && !exchanged) lds_barrier();
  }
  __device__ __forceinline__ float total(float x) const { return waves ? sum16(x) : x; }  // of the waves' values
};

// Mean (0 under RMS) and 1 / standard deviation of a row, from two values of each wave: its own mean, and its squares about that.
// Those of the waves are put together by: squares about the row's mean = theirs + count * (their mean - the row's)^2.  So it takes
// one exchange between waves, and nothing cancels where the mean is large.  Counts: entries of a row in this wave, and in wave
// threadIdx.x % 16.
struct Counts {
  float mine_inv, other;
};
struct Stats {
  float mean, rstd;
};
template <Spread S>
__device__ __forceinline__ f32x2 wave_stats(const float* x, const Columns<S>& col, int kind, const Counts& counts) {
  float mean = 0.f;
  if (kind == LITE_ATTN_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      s += has_tail(S) ? col.part(e, x[e]) : x[e];  // (0 where there is no column)
    mean = sum64(s) * counts.mine_inv;
  }
  float sq = 0.f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const float d = col.part(e, x[e] - mean);
    sq += d * d;
  }
  return f32x2{mean, sum64(sq)};
}
__device__ __forceinline__ Stats row_stats(const Team& team, f32x2 w, int kind, float eps, float inv_D, const Counts& counts) {
  float mean = w[0];
  if (team.waves && kind == LITE_ATTN_NORM_LAYER) {
    mean = sum16(w[0] * counts.other) * inv_D;
    const float d = w[0] - mean;
    w[1] += counts.other * d * d;
  }
  return {mean, rsqrtf(team.total(w[1]) * inv_D + eps)};
}
// Sums that the gradient d of a norm's result asks for, over this wave: of d, and of d (x - mean).
template <Spread S>
__device__ __forceinline__ f32x2 wave_dots(const float* d, const float* x, float mean, const Columns<S>& col) {
  f32x2 s = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const float t = col.part(e, d[e]);
    s[0] += t;
    s[1] += t * (has_tail(S) ? col.part(e, x[e] - mean) : x[e] - mean);
  }
  return f32x2{sum64(s[0]), sum64(s[1])};
}

// The workgroup's share of the rows of a group.
struct Share {
  int batch, group, n0, end, step;  // group of the batch entry; rows n0, n0 + step, ... below end
  __device__ __forceinline__ explicit Share(const ResidualParams& p) {
    const int g = (int)blockIdx.x / p.shares;
    batch = g / p.groups;
    group = g - batch * p.groups;
    n0 = group * p.per_mod + ((int)blockIdx.x - g * p.shares);
    end = min(p.N, (group + 1) * p.per_mod);
    step = p.shares;
  }
  __device__ __forceinline__ Walk walk(const Lines& l, int bytes) const {
    return Walk{l.data + batch * l.stride_b + n0 * l.stride_n, step * l.stride_n, l.data ? bytes : 0};
  }
};

template <Spread S>
__device__ __forceinline__ Counts count_columns(const ResidualParams& p, const Columns<S>& col, float* in_waves) {
  float mine = 0.f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) mine += col.part(e, 1.f);
  mine = sum64(mine);
  if ((threadIdx.x & 63) == 0) in_waves[threadIdx.x >> 6] = mine;
  lds_barrier();
  const int w = threadIdx.x & 15;
  return {1.f / mine, w < (int)(blockDim.x >> 6) ? in_waves[w] : 0.f};
}

template <class KindX, class KindY, Spread S>
__global__ __launch_bounds__(S == kOnes ? 64 : kMaxTeam) void residual_fwd_kernel(const ResidualParams p) {
  __shared__ WaveRoom<3> room;
  __shared__ float in_waves[kMaxTeam / 64];
  touch_arguments<sizeof(ResidualParams)>();
  const Share share(p);
  if (share.n0 >= share.end) return;  // (a group of fewer rows than shares)
  const Columns<S> col((int)threadIdx.x, (int)blockDim.x, p.D);
  Team team = {blockDim.x > 64, 0, &room};
  const int row_x = p.D * Piece<KindX>::kSize, row_y = p.D * Piece<KindY>::kSize;

  Walk x_in = share.walk(p.x, row_x), y_in = share.walk(p.y, row_y);
  Walk x_to = share.walk(p.x_out, row_x), h_to = share.walk(p.h, row_y);
  Piece<KindX> next_x;
  Piece<KindY> next_y;
  auto fetch_next = [&](bool there) {
    load_row(x_in.row_if(there), col, next_x);
    load_row(y_in.row_if(there), col, next_y);
    x_in.step();
    y_in.step();
  };
  fetch_next(true);
  const Counts counts = count_columns(p, col, in_waves);
  float open[kEach], mul[kEach], add[kEach];  // x_out = x + open * norm(y);  h = norm(x_out) * mul + add
  {
    float t[kEach];
    load_mod(p.gate, p.param_dtype, share.batch, share.group, col, open, 1.f);
    load_params(p.post_w, p.param_dtype, col, t, 1.f);
#pragma unroll
    for (int e = 0; e < kEach; ++e) open[e] *= p.alpha * t[e];
    load_params(p.pre_w, p.param_dtype, col, mul, 1.f);
    load_params(p.pre_b, p.param_dtype, col, add, 0.f);
    load_mod(p.scale, p.param_dtype, share.batch, share.group, col, t, 0.f);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      mul[e] *= 1.f + t[e];
      add[e] *= 1.f + t[e];
    }
    load_mod(p.shift, p.param_dtype, share.batch, share.group, col, t, 0.f);
#pragma unroll
    for (int e = 0; e < kEach; ++e) add[e] += t[e];
  }
  no_stores<kRowAccesses<KindX, S> + kRowAccesses<KindY, S>>(x_to);
  for (int n = share.n0; n < share.end; n += share.step) {
    const Piece<KindX> px = next_x;
    const Piece<KindY> py = next_y;
    fetch_next(n + share.step < share.end);
    const bool post = p.y.data && p.post != LITE_ATTN_NORM_NONE, pre = p.h.data && p.pre != LITE_ATTN_NORM_NONE;
    team.meet<S>(pre || post);
    float x[kEach];
    px.unpack(x);
    if (p.y.data) {
      float y[kEach];
      py.unpack(y);
      if (post) {
        f32x2 w[1] = {wave_stats(y, col, p.post, counts)};
        team.exchange(w);
        const Stats s = row_stats(team, w[0], p.post, p.post_eps, p.inv_D, counts);
#pragma unroll
        for (int e = 0; e < kEach; ++e) y[e] = (y[e] - s.mean) * s.rstd;
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e) x[e] += open[e] * y[e];
    }
    store_row<KindX>(x_to.row(), col, x);
    x_to.step();
    if (p.h.data) {
      if (pre) {
        f32x2 w[1] = {wave_stats(x, col, p.pre, counts)};
        team.exchange(w);
        const Stats s = row_stats(team, w[0], p.pre, p.pre_eps, p.inv_D, counts);
#pragma unroll
        for (int e = 0; e < kEach; ++e) x[e] = (x[e] - s.mean) * s.rstd;
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e) x[e] = x[e] * mul[e] + add[e];
    }
    store_row<KindY>(h_to.row(), col, x);
    h_to.step();
  }
}

// Backwards, for a row: with n = pre(x), da = dh (1 + scale), dn = da pre_w
//   dx = dx_out + rstd (dn - mean(dn) [LAYER] - n mean(dn n))
//   dy = the same of dp post_w, dp = alpha gate dx, with n_y = post(y)
// and over the tokens of a row of modulation A = sum dh n, S = sum dh, C = sum dx n_y, from which all six gradients of the
// parameters follow (group_sums_kernel): three sums in registers, where each gradient by itself would need six.  The waves meet
// once for x, with both rows' statistics and the sums of dn and of dn (x - the wave's mean), which those of the waves are put
// together from like the squares, and once more for y: us at 2 x 3913 rows of 1111, four meetings -> two, 56.5 -> 54.4.
template <class KindX, class KindY, Spread S>
__global__ __launch_bounds__(S == kOnes ? 64 : kMaxTeam) void residual_bwd_kernel(const ResidualParams p) {
  __shared__ WaveRoom<3> room;
  __shared__ float in_waves[kMaxTeam / 64];
  touch_arguments<sizeof(ResidualParams)>();
  const Share share(p);
  if (share.n0 >= share.end) return;  // (a group of fewer rows than shares)
  const Columns<S> col((int)threadIdx.x, (int)blockDim.x, p.D);
  Team team = {blockDim.x > 64, 0, &room};
  const int row_x = p.D * Piece<KindX>::kSize, row_y = p.D * Piece<KindY>::kSize;

  Walk x_in = share.walk(p.x, row_x), dh_in = share.walk(p.dh, row_y);
  Walk dxo_in = share.walk(p.dxo, row_x), y_in = share.walk(p.y, row_y);
  Walk dx_to = share.walk(p.dx, row_x), dy_to = share.walk(p.dy, row_y);
  Piece<KindX> next_x, dxo;
  Piece<KindY> next_dh, next_y;
  auto fetch_next = [&](bool there) {
    load_row(x_in.row_if(there), col, next_x);
    load_row(dh_in.row_if(there), col, next_dh);
    load_row(y_in.row_if(there), col, next_y);
    x_in.step();
    dh_in.step();
    y_in.step();
  };
  fetch_next(true);
  const Counts counts = count_columns(p, col, in_waves);
  float open[kEach], mul[kEach];  // alpha gate post_w, (1 + scale) pre_w
  float sum_a[kEach], sum_s[kEach], sum_c[kEach];
  {
    float t[kEach];
    load_mod(p.gate, p.param_dtype, share.batch, share.group, col, open, 1.f);
    load_params(p.post_w, p.param_dtype, col, t, 1.f);
#pragma unroll
    for (int e = 0; e < kEach; ++e) open[e] *= p.alpha * t[e];
    load_params(p.pre_w, p.param_dtype, col, mul, 1.f);
    load_mod(p.scale, p.param_dtype, share.batch, share.group, col, t, 0.f);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      mul[e] *= 1.f + t[e];
      sum_a[e] = sum_s[e] = sum_c[e] = 0.f;
    }
  }
  no_stores<kRowAccesses<KindX, S> + kRowAccesses<KindY, S>>(dx_to);
  for (int n = share.n0; n < share.end; n += share.step) {
    // what the row needs first is asked for a row ahead, the rest now
    const Piece<KindX> px = next_x;
    const Piece<KindY> pdh = next_dh, py = next_y;
    load_row(dxo_in.row(), col, dxo);
    dxo_in.step();
    fetch_next(n + share.step < share.end);
    const bool pre = p.dh.data && p.pre != LITE_ATTN_NORM_NONE, post = p.y.data && p.post != LITE_ATTN_NORM_NONE;
    team.meet<S>(pre || post);
    float dx[kEach], x[kEach], y[kEach];
    px.unpack(x);
    py.unpack(y);
    pdh.unpack(dx);  // (0 if there is no dh)
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      sum_s[e] += dx[e];
      if (!pre && p.dh.data) sum_a[e] += dx[e] * x[e];
    }
    float dh[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      dh[e] = dx[e];
      dx[e] *= mul[e];
    }
    f32x2 w[3] = {};
    if (pre) {
      w[0] = wave_stats(x, col, p.pre, counts);
      w[1] = wave_dots(dx, x, w[0][0], col);
    }
    if (post) w[2] = wave_stats(y, col, p.post, counts);
    if (pre || post) team.exchange(w);
    float rstd = 1.f;
    if (post) {
      const Stats s = row_stats(team, w[2], p.post, p.post_eps, p.inv_D, counts);
      rstd = s.rstd;
#pragma unroll
      for (int e = 0; e < kEach; ++e) y[e] = (y[e] - s.mean) * rstd;
    }
    if (pre) {
      const Stats s = row_stats(team, w[0], p.pre, p.pre_eps, p.inv_D, counts);
      const float mean = p.pre == LITE_ATTN_NORM_LAYER ? team.total(w[1][0]) * p.inv_D : 0.f;
      const float pull = team.total(w[1][1] + (w[0][0] - s.mean) * w[1][0]) * s.rstd * p.inv_D;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        x[e] = (x[e] - s.mean) * s.rstd;
        sum_a[e] += dh[e] * x[e];
        dx[e] = s.rstd * (dx[e] - mean - x[e] * pull);
      }
    }
    float more[kEach];
    dxo.unpack(more);
#pragma unroll
    for (int e = 0; e < kEach; ++e) dx[e] += more[e];
    store_row<KindX>(dx_to.row(), col, dx);
    dx_to.step();
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      sum_c[e] += dx[e] * y[e];
      dx[e] *= open[e];
    }
    if (post && p.dy.data) {
      f32x2 d[1] = {wave_dots(dx, y, 0.f, col)};
      team.exchange(d);
      const float mean = p.post == LITE_ATTN_NORM_LAYER ? team.total(d[0][0]) * p.inv_D : 0.f;
      const float pull = team.total(d[0][1]) * p.inv_D;
#pragma unroll
      for (int e = 0; e < kEach; ++e) dx[e] = rstd * (dx[e] - mean - y[e] * pull);
    }
    store_row<KindY>(dy_to.row(), col, dx);
    dy_to.step();
  }
  if (!p.part) return;
  const int64_t bytes = 4 * (int64_t)p.D;
  Walk sums = {reinterpret_cast<char*>(p.part) + 3 * bytes * blockIdx.x, bytes, (int)bytes};
  store_row<F32>(sums.row(), col, sum_a);
  sums.step();
  store_row<F32>(sums.row(), col, sum_s);
  sums.step();
  store_row<F32>(sums.row(), col, sum_c);
}

// Sums of a row of modulation: its shares' sums in order, kColumns threads an equal part of them, and what follows from them.
// If the group is the only one, its parts of the weights' gradients are these gradients.
template <int kColumns>  // that a workgroup takes
__global__ __launch_bounds__(1024) void group_sums_kernel(const ResidualParams p, int all_groups) {
  __shared__ float sums[1024 / kColumns][3][kColumns];
  const int lane = threadIdx.x % kColumns, part = threadIdx.x / kColumns, parts = blockDim.x / kColumns;
  const int column = blockIdx.y * kColumns + lane;
  const size_t D = p.D;
  for (int group = blockIdx.x; group < all_groups; group += gridDim.x) {
    const int b = group / p.groups, g = group - b * p.groups;
    const int shares = min(p.shares, min(p.N, (g + 1) * p.per_mod) - g * p.per_mod);
    const int from = part_start(shares, parts, part), to = part_start(shares, parts, part + 1);
    float a = 0.f, s = 0.f, c = 0.f;
    if (column < p.D) {
      const float* at = p.part + ((size_t)group * p.shares + from) * 3 * D + column;
#pragma unroll 4
      for (int x = from; x < to; ++x, at += 3 * D) {
        a += at[0];
        s += at[D];
        c += at[2 * D];
      }
    }
    sums[part][0][lane] = a;
    sums[part][1][lane] = s;
    sums[part][2][lane] = c;
    __syncthreads();
    if (part == 0 && column < p.D) {
      for (int w = 1; w < parts; ++w) {
        a += sums[w][0][lane];
        s += sums[w][1][lane];
        c += sums[w][2][lane];
      }
      const int d = p.param_dtype;
      const size_t at = (size_t)group * D + column;
      const float post_w = p.post_w ? load_param(p.post_w, d, column) : 1.f;
      const float pre_w = p.pre_w ? load_param(p.pre_w, d, column) : 1.f;
      auto mod = [&](const Lines& l, float missing) {
        return l.data ? load_param(l.data + b * l.stride_b + g * l.stride_n, d, column) : missing;
      };
      const float gate = mod(p.gate, 1.f), open = 1.f + mod(p.scale, 0.f);
      if (p.dgate) p.dgate[at] = p.alpha * post_w * c;
      if (p.dscale) p.dscale[at] = pre_w * a + (p.pre_b ? load_param(p.pre_b, d, column) * s : 0.f);
      if (p.dshift) p.dshift[at] = s;
      const bool only = all_groups == 1;
      float* const to_w[3] = {p.dpre_w, p.dpre_b, p.dpost_w};
      const float w[3] = {open * a, open * s, p.alpha * gate * c};
#pragma unroll
      for (int x = 0; x < 3; ++x)
        if (to_w[x]) (only ? to_w[x] : p.group_sums + ((size_t)group * 3 + x) * D)[column] = w[x];
    }
    __syncthreads();
  }
}

// Gradients of pre_weight, pre_bias and post_weight: the groups' parts in order.
__global__ __launch_bounds__(1024) void weight_sums_kernel(const ResidualParams p, int all_groups) {
  __shared__ float sums[16][64];
  float* const out = blockIdx.y == 0 ? p.dpre_w : blockIdx.y == 1 ? p.dpre_b : p.dpost_w;
  if (!out) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int column = blockIdx.x * 64 + lane;
  const int from = part_start(all_groups, 16, wave), to = part_start(all_groups, 16, wave + 1);
  float sum = 0.f;
  if (column < p.D) {
    const float* part = p.group_sums + blockIdx.y * (size_t)p.D + column;
#pragma unroll 8
    for (int x = from; x < to; ++x) sum += part[(size_t)x * 3 * p.D];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && column < p.D) {
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    out[column] = sum;
  }
}

template <class Kind, bool HALVES, bool WHOLE, bool BWD>
void launch_rotary_sums(const RotaryParams& p, const LayerLaunch& l, hipStream_t st) {
  if (l.sums == kSumNone)
    rotary_kernel<Kind, HALVES, WHOLE, kSumNone, BWD><<<l.blocks, l.threads, 0, st>>>(p);
  else if (l.sums == kSumLanes)
    rotary_kernel<Kind, HALVES, WHOLE, kSumLanes, BWD><<<l.blocks, l.threads, 0, st>>>(p);
  else if (l.sums == kSumHeads)
    rotary_kernel<Kind, HALVES, WHOLE, kSumHeads, BWD><<<l.blocks, l.threads, 0, st>>>(p);
  else
    rotary_kernel<Kind, HALVES, WHOLE, kSumWaves, BWD><<<l.blocks, l.threads, 0, st>>>(p);
}
template <class Kind, bool BWD>
void launch_rotary_way(const RotaryParams& p, const LayerLaunch& l, hipStream_t st) {
  const bool whole = p.head_dim % kEach == 0 && (!p.halves || p.pairs % 4 == 0);
  if (p.halves)
    whole ? launch_rotary_sums<Kind, true, true, BWD>(p, l, st) : launch_rotary_sums<Kind, true, false, BWD>(p, l, st);
  else
    whole ? launch_rotary_sums<Kind, false, true, BWD>(p, l, st) : launch_rotary_sums<Kind, false, false, BWD>(p, l, st);
}
template <class Kind>
void launch_rotary_kind(const RotaryParams& p, const LayerLaunch& l, bool bwd, hipStream_t st) {
  bwd ? launch_rotary_way<Kind, true>(p, l, st) : launch_rotary_way<Kind, false>(p, l, st);
}

template <class KindX, class KindY, Spread S>
void launch_residual_way(const ResidualParams& p, const LayerLaunch& l, bool bwd, hipStream_t st) {
  if (bwd)
    residual_bwd_kernel<KindX, KindY, S><<<l.blocks, l.threads, 0, st>>>(p);
  else
    residual_fwd_kernel<KindX, KindY, S><<<l.blocks, l.threads, 0, st>>>(p);
}
template <class KindX, class KindY>
void launch_residual_kind(const ResidualParams& p, const LayerLaunch& l, bool bwd, hipStream_t st) {
  constexpr bool kWide = Piece<KindX>::kSize == 4;
  if (p.D % kEach == 0)
    launch_residual_way<KindX, KindY, kWide ? kFours : kEights>(p, l, bwd, st);
  else if (p.D > kEach)
    launch_residual_way<KindX, KindY, kWide ? kFoursTail : kEightsTail>(p, l, bwd, st);
  else
    launch_residual_way<KindX, KindY, kOnes>(p, l, bwd, st);
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, const LayerLaunch& l, int dtype, bool bwd, hipStream_t st) {
  if (dtype == LITE_ATTN_BF16)
    launch_rotary_kind<Bf16>(p, l, bwd, st);
  else if (dtype == LITE_ATTN_F16)
    launch_rotary_kind<F16>(p, l, bwd, st);
  else
    launch_rotary_kind<F32>(p, l, bwd, st);
  return hipGetLastError();
}

// The shares' sums -> the gradients of the weights of q and k, as far as they are wanted.
hipError_t launch_rotary_weights(const RotaryParams& p, float* dq_weight, float* dk_weight, hipStream_t st) {
  RowSums s;
  float* const out[2] = {dq_weight, dk_weight};
  int blocks[2];
  for (int x = 0; x < 2; ++x) {
    const bool row = p.by_row;
    s.part[x] = p.side[x].part;
    s.out[x] = out[x];
    s.columns[x] = out[x] ? (row ? p.side[x].heads : 1) * p.head_dim : 0;
    s.rows[x] = p.N == 0 ? 0 : p.batch * p.shares * (row ? p.tokens : p.groups);
    blocks[x] = (s.columns[x] + 63) / 64;
  }
  s.blocks0 = blocks[0];
  if (blocks[0] + blocks[1] == 0) return hipSuccess;
  sum_rows_kernel<<<blocks[0] + blocks[1], 1024, 0, st>>>(s);
  return hipGetLastError();
}

hipError_t launch_residual(const ResidualParams& p, const LayerLaunch& l, int dtype, int stream_dtype, bool bwd,
                           hipStream_t st) {
  if (dtype == LITE_ATTN_F32)
    launch_residual_kind<F32, F32>(p, l, bwd, st);
  else if (dtype == LITE_ATTN_BF16 && stream_dtype == LITE_ATTN_BF16)
    launch_residual_kind<Bf16, Bf16>(p, l, bwd, st);
  else if (dtype == LITE_ATTN_BF16)
    launch_residual_kind<F32, Bf16>(p, l, bwd, st);
  else if (stream_dtype == LITE_ATTN_F16)
    launch_residual_kind<F16, F16>(p, l, bwd, st);
  else
    launch_residual_kind<F32, F16>(p, l, bwd, st);
  return hipGetLastError();
}

hipError_t launch_residual_sums(const ResidualParams& p, hipStream_t st) {
  const int64_t groups = (int64_t)p.batch * p.groups;
  if (groups > 0) {
    const int waves = p.shares < 2 ? 1 : p.shares < 32 ? 4 : 16;
    // Few workgroups of 64 columns do not get the shares' sums in fast enough: us at 200000 rows of 128, 64 -> 32 columns 155 ->
    // 139, 60000 of 1111 214 -> 207, 2 x 1000 of 1536 21.0 -> 20.5; but 8 groups of 1111 51.6 -> 55, 21 of 1536 173 -> 184.
    const bool few = groups * ((p.D + 63) / 64) < 64;
    const int columns = few ? 32 : 64;
    const dim3 grid((unsigned)(groups < 65536 ? groups : 65536), (unsigned)((p.D + columns - 1) / columns));
    if (few)
      group_sums_kernel<32><<<grid, 64 * waves, 0, st>>>(p, (int)groups);
    else
      group_sums_kernel<64><<<grid, 64 * waves, 0, st>>>(p, (int)groups);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (groups != 1 && (p.dpre_w || p.dpre_b || p.dpost_w))
    weight_sums_kernel<<<dim3((unsigned)(p.D + 63) / 64, 3), 1024, 0, st>>>(p, (int)groups);
  return hipGetLastError();
}

}  // namespace la

extern "C" {

int lite_attn_rotary_fwd(const lite_attn_rotary_desc_t* desc, const lite_attn_rotary_fwd_t* args, void* hip_stream) {
  int rc = la::check_rotary(desc);
  if (rc != LITE_ATTN_OK) return rc;
  if (!args) return LITE_ATTN_EINVAL;
  if (desc->seqlen == 0) return LITE_ATTN_OK;
  la::RotaryParams p;
  la::LayerLaunch l;
  rc = la::plan_rotary(*desc, *args, &p, &l);
  if (rc != LITE_ATTN_OK) return rc;
  const hipError_t e = la::launch_rotary(p, l, desc->dtype, false, reinterpret_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? LITE_ATTN_OK : la::hip_fail(e);
}

int lite_attn_rotary_bwd(const lite_attn_rotary_desc_t* desc, const lite_attn_rotary_bwd_t* args, void* hip_stream) {
  int rc = la::check_rotary(desc);
  if (rc != LITE_ATTN_OK) return rc;
  if (!args) return LITE_ATTN_EINVAL;
  la::RotaryParams p;
  la::LayerLaunch l;
  rc = la::plan_rotary(*desc, *args, &p, &l);
  if (rc != LITE_ATTN_OK) return rc;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  if (desc->seqlen > 0) e = la::launch_rotary(p, l, desc->dtype, true, stream);
  if (e == hipSuccess && (args->dq_weight || args->dk_weight))
    e = la::launch_rotary_weights(p, args->dq_weight, desc->heads_k ? args->dk_weight : nullptr, stream);
  return e == hipSuccess ? LITE_ATTN_OK : la::hip_fail(e);
}

int lite_attn_residual_norm_fwd(const lite_attn_residual_desc_t* desc, const lite_attn_residual_fwd_t* args,
                                void* hip_stream) {
  int rc = la::check_residual(desc);
  if (rc != LITE_ATTN_OK) return rc;
  if (!args) return LITE_ATTN_EINVAL;
  if (desc->seqlen == 0) return LITE_ATTN_OK;
  la::ResidualParams p;
  la::LayerLaunch l;
  rc = la::plan_residual(*desc, *args, &p, &l);
  if (rc != LITE_ATTN_OK) return rc;
  const hipError_t e =
      la::launch_residual(p, l, desc->dtype, desc->stream_dtype, false, reinterpret_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? LITE_ATTN_OK : la::hip_fail(e);
}

int lite_attn_residual_norm_bwd(const lite_attn_residual_desc_t* desc, const lite_attn_residual_bwd_t* args,
                                void* hip_stream) {
  int rc = la::check_residual(desc);
  if (rc != LITE_ATTN_OK) return rc;
  if (!args) return LITE_ATTN_EINVAL;
  la::ResidualParams p;
  la::LayerLaunch l;
  rc = la::plan_residual(*desc, *args, &p, &l);
  if (rc != LITE_ATTN_OK) return rc;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  if (desc->seqlen > 0) e = la::launch_residual(p, l, desc->dtype, desc->stream_dtype, true, stream);
  if (e == hipSuccess && p.part) e = la::launch_residual_sums(p, stream);
  return e == hipSuccess ? LITE_ATTN_OK : la::hip_fail(e);
}

}  // extern "C"
