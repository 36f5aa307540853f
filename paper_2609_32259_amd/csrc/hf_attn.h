// Device helpers shared by the attention kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cfloat>

#include "hf_internal.h"

namespace hf {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4_t;

#define FI __device__ __forceinline__

// A row's running maximum starts at the least finite value rather than at
// -infinity, so that exp2(s - m) of a row that has seen no key is exp2(-inf) = 0.
constexpr float kNoMax = -FLT_MAX;

// The maximum that a row's weights are formed against is raised only when a new
// score passes it by more than this (in powers of two): until then weights of up
// to 2^8 are as exact as those of at most 1, in fp32 sums and in bf16 operands
// alike, and the sums need no rescaling.  Most steps skip it.
constexpr float kRaise = 8.0f;

// Scores far from 0.  A weight is 2^(s c - m), formed by one fused multiply-add, and m the
// rounded product top * c of the row's largest score.  From 2^31 on its rounding alone is up
// to 2^7 and more, and every weight of the row may overflow or vanish.  From 2^30 on a row
// therefore multiplies by the power of two below c, which makes m exact.  Its softmax stays the
// same: there two scores differ by 2^6 at least in units of c, by 2^5 in the other's, and all
// weights but the largest scores' are below the rounding of their sum in either.
// A unit for each row, in a vector register, costs the dense loops 1% (8,192 tokens 487 -> 491
// us), so they have c, and a row that ends far away is computed in the second pass.  The paged
// kernel, which has none, keeps a unit for each row (16 sequences of 4 to 8K tokens 25.4 -> 25.7
// us; a second pass there measured the same).
constexpr float kFar = 0x1p30f;
FI bool far_max(float m) { return !(fabsf(m) < kFar); }  // (kNoMax is: c times a score may lie below it)
FI float far_unit(float c) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, c) & 0x7f800000u); }

// Raises a row's maximum m, in units of cr, to that of its largest score `top` where that
// passes it, and returns the factor for what was summed (0 where the unit changes: then all of
// it is as far away).  units: cr may become far_unit(c).
FI float raise(float top, float c, bool units, float& cr, float& m) {
  if (!(top * cr > m + kRaise)) return 1.0f;
  float now = c, to = top * c;
  if (units && far_max(to)) {
    now = far_unit(c);
    to = top * now;
  }
  const float f = now == cr ? __builtin_amdgcn_exp2f(m - to) : 0.0f;
  cr = now;
  m = to;
  return f;
}

// The maximum that a row of weight l ends with, in units of c, which is what it is joined to
// others by.  Where it saw keys and all their scores were -infinity it is that (weights 0/0,
// whose result is NaN); kNoMax stays for a row that saw none (result 0).  l is 0 for these
// two alone.
FI float end_max(float m, float cr, float c, float l, bool saw) {
  if (l == 0.0f) return saw ? -INFINITY : kNoMax;
  return cr == c ? m : fminf(fmaxf(m / cr * c, -FLT_MAX), FLT_MAX);
}

// s_waitcnt immediate that waits until at most n vector-memory operations are
// outstanding and leaves the other counters alone (gfx9 encoding).
constexpr int wait_vm_only(int n) { return (n & 0xF) | ((n >> 4) << 14) | (7 << 4) | (0xF << 8); }
// All vector-memory and LDS operations; the LDS operations alone.
constexpr int kWaitMemory = 7 << 4;
constexpr int kWaitLds = 0xF | (3 << 14) | (7 << 4);

// A buffer resource of `bytes` from a pointer that every lane holds.
FI __amdgpu_buffer_rsrc_t buffer_at(const void* p, int bytes) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(((uint64_t)hi << 32) | lo), 0, __builtin_amdgcn_readfirstlane(bytes),
                                           0x00020000);
}

FI uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// A buffer load of 16 bytes a lane from p + off (within `bytes`) to LDS (to + 16 lane), which the
// compiler counts neither as a load nor as an LDS access: only explicit waits order it.
FI void load_lds_unseen(const void* p, int bytes, int off, void* to) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  const u32x4 rsrc = {lo, hi & 0xffffu, (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_addr(to))), "v"(off), "s"(rsrc)
               : "memory", "m0");
}

FI uint32_t pack_bf16(float a, float b) {
  bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

FI bool finite_bits(float x) {
  return (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) != 0x7f800000u;
}

// max and sum of a register over the lanes l ^ 32, and l ^ 16 (exchanges of half-waves
// and of 16-lane rows, without LDS).
FI float max_xor32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];  // (copies: a bit cast of an element itself takes element 0)
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
FI float add_xor32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
FI float max_xor16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];  // (copies: a bit cast of an element itself takes element 0)
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
FI float add_xor16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

FI int divide(int n, const Divide& d) {
  return (int)(((uint64_t)(uint32_t)n * d.magic) >> d.shift);
}

// The sequence that item i of a prefix array (a member of the sequences' records)
// belongs to: a lane looks at each (at most HF_MAX_BATCH = 64), where a walk would
// wait for memory once a step.
static_assert(HF_MAX_BATCH <= 64, "one lane a sequence");
template <class S>
FI int find_seq(const S* q, int32_t S::*first, int B, int i) {
  if (B == 1) return 0;
  const int lane = threadIdx.x & 63;
  const bool before = lane < B && q[lane].*first <= i;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)) - 1);
}

// Elements to a sequence's first row.
FI long long seq_at(int b, int rows_before, long long sb, long long st) {
  return sb == -1 ? rows_before * st : b * sb;
}

// The work item of this workgroup: its head, sequence, row tile and part.  Heads
// vary fastest, so that with 8 heads the workgroups of one head, which read the
// same keys, run on one XCD (workgroup i runs on XCD i % 8) and share them in its
// L2.  Row tiles run from the last to the first: a causal tile's work grows with
// its rows, and the long ones go first.
struct AttnItem {
  int b, h, tile, part;
  int n, t, rows;           // query tokens, keys, query rows of a head (n G < 2^31: host check)
  int row0, key0, parts, part0;
};
FI AttnItem attn_item(const AttnSeqs& s, int tile_rows) {
  AttnItem it;
  const int wg = blockIdx.x;
  int i = divide(wg, s.by_h);
  it.h = wg - i * s.H;
  // Where a CU runs several workgroups at once, which it gets in rounds of one a CU,
  // every other round turns, so that long tiles are joined by short ones.
  if (s.snake) {
    const int r = i / s.snake;
    if (r & 1) i = min(s.n_items, (r + 1) * s.snake) - 1 - (i - r * s.snake);
  }
  it.b = find_seq(s.q, &AttnSeq::item0, s.B, i);
  const AttnSeq q = s.q[it.b];
  it.n = q.n;
  it.t = q.t;
  it.rows = q.n * s.G;
  it.row0 = q.row0;
  it.key0 = q.key0;
  it.parts = q.parts;
  it.part0 = q.part0;
  i -= q.item0;
  it.part = 0;
  if (q.parts > 1) {
    const int x = i / q.parts;
    it.part = i - x * q.parts;
    i = x;
  }
  it.tile = (it.rows + tile_rows - 1) / tile_rows - 1 - i;
  return it;
}

// The last key a row sees (-1: none), from its token.
FI int last_key(const AttnSeqs& s, const AttnItem& it, int token) {
  return s.causal ? min(it.t - 1, token + it.t - it.n) : it.t - 1;
}

// Where a row's result goes, and its log-sum-exp.
FI long long out_at(const AttnIO& io, const AttnSeqs& s, const AttnItem& it, int token, int head) {
  return seq_at(it.b, it.row0, io.o_sb, io.o_st) + token * io.o_st + head * io.o_sh;
}
FI void write_lse(const AttnIO& io, const AttnSeqs& s, const AttnItem& it, int token, int head,
                  float m, float l) {
  if (io.lse)
    io.lse[(long long)(it.row0 + token) * (s.H * s.G) + head] =
        l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}
FI float inverse_weight(float m, float l) { return l == 0.0f && m == kNoMax ? 0.0f : 1.0f / l; }
FI long long part_slot(const AttnItem& it, int r) {
  return it.part0 + ((long long)it.h * it.rows + r) * it.parts + it.part;
}

// Where four waves share R query rows and deal the keys among them: their sums, each
// against the waves' common maximum, lie in LDS as [wave][row][channel] with 16-byte
// chunk x of row r at slot x ^ (r % 16), so that the 16 rows that a write touches at
// once lie on distinct banks.  Each thread adds four channels of a row and writes the
// result, or the part.  sm, sl: the waves' maxima and weights.
template <int R, int D>
FI int sum_slot(int wave, int r, int chunk) {
  return (wave * R + r) * (D / 4) + (chunk ^ (r & 15));
}
template <int R, int D, int NW, bool F32>
FI void write_joined(const AttnIO& io, const AttnSeqs& s, const AttnItem& it, int row0,
                     const f32x4* sums, const float (&sm)[NW][R], const float (&sl)[NW][R]) {
  const int rows = min(R, it.rows - row0);
  for (int at = threadIdx.x; at < rows * (D / 4); at += 64 * NW) {
    const int rl = at / (D / 4), ch = at % (D / 4), r = row0 + rl;
    float m = kNoMax, least = kNoMax, l = 0.0f;
    f32x4 v = {};
#pragma unroll
    for (int y = 0; y < NW; ++y) {
      m = fmaxf(m, sm[y][rl]);
      least = fminf(least, sm[y][rl]);
    }
#pragma unroll
    for (int y = 0; y < NW; ++y) {
      v += sums[sum_slot<R, D>(y, rl, ch)];
      l = fmaf(sl[y][rl], __builtin_amdgcn_exp2f(sm[y][rl] - m), l);
    }
    if (l == 0.0f) m = least;  // (-infinity if some wave saw keys)
    if (it.parts == 1) {
      const int token = divide(r, s.by_g), head = it.h * s.G + r - token * s.G;
      const long long to = out_at(io, s, it, token, head) + 4 * ch;
      v *= inverse_weight(m, l);
      if (F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(io.out) + to) = v;
      } else {
        const u32x2 x = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(io.out) + to) = x;
      }
      if (ch == 0) write_lse(io, s, it, token, head, m, l);
    } else {
      const long long slot = part_slot(it, r);
      *reinterpret_cast<f32x4*>(io.part + slot * D + 4 * ch) = v;
      if (ch == 0) {
        io.ml[2 * slot] = m;
        io.ml[2 * slot + 1] = l;
      }
    }
  }
}

}  // namespace hf
