// A paged cache held in 4 bits: appending rows, reading them back, and attention
// over it (the format stands in heterofold.h).
//
// Attention.  With the codes c and a group's scale s and offset o,
//
//   <q, k_t> = sum_g [ s_tg <q_g, c_tg> + o_tg sum(q_g) ]
//   out_g    = sum_t (p_t s_tg) c_tg + sum_t p_t o_tg
//
// where g runs over the groups of 32 channels.  A group is the reduction length of
// v_mfma_f32_16x16x32_bf16, so one instruction gives <q_g, c_tg> of 16 tokens and 16
// rows, and the codes are exact in bf16: a code moved into the mantissa under the
// exponent of 16 is 16 + code.  That costs a shift and an and-or for two codes, and
// the 16s are taken out again with numbers that are needed anyway (o - 16 s, and a
// product of the weights with 1).  Scales and offsets are applied in fp32.
#include <hip/hip_runtime.h>

#include "hf_attn.h"
#include "hf_paged.h"

namespace hf {
namespace {

// ---------------------------------------------------------------------------
// Rows in and out.  A workgroup takes a block of 32 tokens (the unit of the value
// codes' order) of one sequence, layer, role and head; 16 channels a thread.
// ---------------------------------------------------------------------------

constexpr int kHeads = 4;  // that a workgroup takes at most

struct RowItem {
  int b, l, h, role;
  int start, pos0, src0;  // the sequence's first token, position offset, rows before it
  int tok0;          // first token of the block
  int lo, hi;        // tokens of the call in it, relative to tok0
  uint8_t* head;     // the head's part of the page, or nullptr (a hole)
  int row0;          // the block's first row in the page
};

template <int D>
FI RowItem row_item(const PagedRowsArgs& a, int hpw) {
  RowItem it;
  const int wg = blockIdx.x, groups = (a.H + hpw - 1) / hpw;
  const int i = divide(wg, a.by_groups);
  it.h = (wg - i * groups) * hpw;
  it.role = blockIdx.y;
  it.l = blockIdx.z;
  it.b = find_seq(a.q, &RowsSeq::blk0, a.B, i);
  const RowsSeq q = a.q[it.b];
  it.start = q.start;
  it.pos0 = q.pos0;
  it.src0 = q.row0;
  it.tok0 = (q.start / 32 + (i - q.blk0)) * 32;
  it.lo = max(q.start - it.tok0, 0);
  it.hi = min(q.start + q.n - it.tok0, 32);
  const int page = a.table[it.b * a.table_stride + (it.tok0 >> a.log2_page)];
  it.row0 = it.tok0 & ((1 << a.log2_page) - 1);
  it.head = nullptr;
  if ((unsigned)page < (unsigned)a.n_pages)
    it.head = a.pages + ((long long)it.l * a.n_pages + page) * a.page_bytes;
  return it;
}

// Elements to the dense row of token tok of the block, head 0.
FI long long rows_at(const PagedRowsArgs& a, const RowItem& it, int tok) {
  const long long sb = it.role == 0 ? a.k_sb : a.v_sb, st = it.role == 0 ? a.k_st : a.v_st;
  return seq_at(it.b, it.src0, sb, st) + it.l * (it.role == 0 ? a.k_sl : a.v_sl) +
         (it.tok0 + tok - it.start) * st;
}

// Eight channels as they are loaded, and their values.
template <class T>
struct Raw8 {
  u32x4 v[sizeof(T) / 2];
  FI void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  FI void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w = sizeof(T) == 4 ? v[i / 4 % (sizeof(T) / 2)][i & 3] : v[0][i / 2];
      x[i] = __builtin_bit_cast(float, sizeof(T) == 4 ? w : i & 1 ? w & 0xffff0000u : w << 16);
    }
  }
};

template <class T>
FI void store8(T* p, const float (&x)[8]);
template <>
FI void store8<uint16_t>(uint16_t* p, const float (&x)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<u32x4*>(p) = v;
}
template <>
FI void store8<float>(float* p, const float (&x)[8]) {
  const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
  reinterpret_cast<f32x4*>(p)[0] = a;
  reinterpret_cast<f32x4*>(p)[1] = b;
}

// Codes and word of a group spread over four lanes (l, l ^ 1, l ^ 2, l ^ 3), eight
// channels a lane.  Codes as a dword, channel j at nibble j.
FI float quad_xor1(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xb1, 0xf, 0xf, true));
}
FI float quad_xor2(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4e, 0xf, 0xf, true));
}
FI uint32_t code_group(const float (&x)[8], uint32_t& word) {
#pragma clang fp contract(off)
  // minimum and maximum pass a NaN on
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) {
    lo = __builtin_elementwise_minimum(lo, x[j]);
    hi = __builtin_elementwise_maximum(hi, x[j]);
  }
  lo = __builtin_elementwise_minimum(lo, quad_xor1(lo));
  hi = __builtin_elementwise_maximum(hi, quad_xor1(hi));
  lo = __builtin_elementwise_minimum(lo, quad_xor2(lo));
  hi = __builtin_elementwise_maximum(hi, quad_xor2(hi));
  const float o = bf16_round(lo);
  float s = bf16_round((hi - lo) / 15.0f);
  if (s < 0x1p-100f) s = 0.0f;
  word = __builtin_bit_cast(uint32_t, s) | (__builtin_bit_cast(uint32_t, o) >> 16);
  float q[8];
  // True quotients: what lies halfway between two codes goes to the even one.  With the
  // rounded reciprocal r of s, q = d r and its remainder d - q s (exact), q + rem r is
  // the rounded quotient, wherever r and the remainder are normal numbers or the
  // quotient rounds to 0; a third of a division's instructions.
  if (s >= 0x1p-100f && s <= 0x1p100f) {
    const float r = 1.0f / s;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = x[j] - o, e = d * r;
      q[j] = __builtin_amdgcn_fmed3f(rintf(fmaf(fmaf(-e, s, d), r, e)), 0.0f, 15.0f);
    }
  } else if (finite_bits(o) && finite_bits(s)) {
    const float div = s > 0.0f ? s : INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = __builtin_amdgcn_fmed3f(rintf((x[j] - o) / div), 0.0f, 15.0f);
  } else {
    word = 0x7fc07fc0u;  // NaN, NaN
    return 0;
  }
  // four codes to a float: whole numbers below 2^16
  const float c0 = fmaf(fmaf(fmaf(q[3], 16.0f, q[2]), 16.0f, q[1]), 16.0f, q[0]);
  const float c1 = fmaf(fmaf(fmaf(q[7], 16.0f, q[6]), 16.0f, q[5]), 16.0f, q[4]);
  return (uint32_t)c0 | ((uint32_t)c1 << 16);
}

// Nibble j of a[t] to nibble t of a[j].
FI void transpose_nibbles(uint32_t (&a)[8]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {  // halves of dwords t and t + 4
    const uint32_t x = a[t], y = a[t + 4];
    a[t] = __builtin_amdgcn_perm(y, x, 0x05040100u);
    a[t + 4] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
#pragma unroll
  for (int t = 0; t < 8; t += 4)
#pragma unroll
    for (int u = t; u < t + 2; ++u) {  // bytes
      const uint32_t x = a[u], y = a[u + 2];
      a[u] = __builtin_amdgcn_perm(y, x, 0x06020400u);
      a[u + 2] = __builtin_amdgcn_perm(y, x, 0x07030501u);
    }
#pragma unroll
  for (int t = 0; t < 8; t += 2) {
    const uint32_t x = a[t], y = a[t + 1];
    a[t] = (x & 0x0f0f0f0fu) | ((y << 4) & 0xf0f0f0f0u);
    a[t + 1] = ((x >> 4) & 0x0f0f0f0fu) | (y & 0xf0f0f0f0u);
  }
}

// cos and sin of pos * w_k for the block's 32 positions, to LDS [32][D/2], fp64
// angles rounded once.  Four chains a channel pair, eight positions each: one sine
// and cosine at the chain's first position, then a complex product with the step's
// (error 8 * 2^-53).  (For blocks of one token, forming its angle alone gains nothing: 4.7 us a
// call either way.)
template <int D>
FI void fill_angles(const PagedRowsArgs& a, const RowItem& it, float2* cs) {
  constexpr int HD = D / 2;
  const int k = threadIdx.x % HD, m = threadIdx.x / HD;  // m < 4
  const double w = a.w[k];
  double c, s, dc, ds;
  sincos(w, &ds, &dc);
  sincos(((double)it.pos0 + it.tok0 + 8 * m) * w, &s, &c);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cs[(8 * m + j) * HD + k] = make_float2((float)c, (float)s);
    const double t = c * dc - s * ds;
    s = s * dc + c * ds;
    c = t;
  }
}

// Bound by HBM: a transfer's cache of 40 layers and 7.3K tokens (1.19 GB in, 0.37 GB out)
// takes 305 to 323 us, 4.8 to 5.1 TB/s (a device copy, which writes as much as it reads,
// reaches 4.7); a token for each of eight sequences 4.8 us, the latency of its loads one after
// another.
// ROT: a call that rotates its keys.  (Their angles take registers and LDS that a call which
// only moves rows would miss for loads in flight: 377 and 365 us at that size with and
// without.)
template <class T, int D, bool ROT>
__global__ __launch_bounds__(2 * D) void paged_append_kernel(const PagedRowsArgs a, const int hpw) {
  constexpr int TPT = D / 16;  // threads a token
  constexpr int G = D / 32, O = D / 8;
  constexpr int LD = O + (D == 128 ? 4 : 2);  // dwords a token in LDS: tokens 4 apart on other banks
  constexpr int NH = kHeads;
  __shared__ float2 cs[ROT ? 32 * D / 2 : 1];
  __shared__ uint32_t codes[NH][32 * LD];
  const RowItem it = row_item<D>(a, hpw);
  if (!it.head) return;
  const int tok = threadIdx.x / TPT, j = threadIdx.x % TPT;
  const bool on = tok >= it.lo && tok < it.hi;
  const bool rot = ROT && it.role == 0;
  const PageHead<D> ph(a.log2_page);
  const int row = it.row0 + tok;
  const T* src = static_cast<const T*>(it.role == 0 ? a.k : a.v) + rows_at(a, it, tok);
  const long long sh = it.role == 0 ? a.k_sh : a.v_sh;
  const int heads = min(hpw, a.H - it.h);
  Raw8<T> r0[NH], r1[NH];  // channels 8 j .. and D/2 + 8 j ..: rotation pairs
  if (on) {  // (a group's four lanes hold the same token)
#pragma unroll
    for (int i = 0; i < NH; ++i)
      if (i < heads) {
        r0[i].load(src + (it.h + i) * sh + 8 * j);
        r1[i].load(src + (it.h + i) * sh + D / 2 + 8 * j);
      }
  }
  if (rot) {  // (while the rows are on their way)
    fill_angles<D>(a, it, cs);
    __syncthreads();
  }
  if (on) {
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      if (i >= heads) break;
      float x0[8], x1[8];
      r0[i].values(x0);
      r1[i].values(x1);
      if (ROT && rot) {
#pragma clang fp contract(off)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 r = cs[tok * (D / 2) + 8 * j + e];
          const float u = x0[e], v = x1[e];
          x0[e] = u * r.x - v * r.y;
          x1[e] = v * r.x + u * r.y;
        }
      }
      uint32_t w0, w1;
      const uint32_t c0 = code_group(x0, w0), c1 = code_group(x1, w1);
      uint8_t* head = it.head + (long long)(it.h + i) * ph.bytes();
      uint32_t* words = reinterpret_cast<uint32_t*>(head + ph.word(it.role, row));
      if ((j & 3) == 0) {
        words[j >> 2] = w0;
        words[G / 2 + (j >> 2)] = w1;
      }
      if (it.role == 0) {
        uint32_t* kc = reinterpret_cast<uint32_t*>(head + ph.kcode(row));
        kc[(j & 3) * G + (j >> 2)] = c0;
        kc[(j & 3) * G + G / 2 + (j >> 2)] = c1;
      } else {
        codes[i][tok * LD + j] = c0;
        codes[i][tok * LD + O / 2 + j] = c1;
      }
    }
  }
  if (it.role == 0) return;
  // Value codes to the order of the block, eight tokens by eight channels a thread.
  // Tokens that are not the call's keep what is there.
  __syncthreads();
  static_assert(NH == 2 * D / (D / 2), "a thread of each head, block quarter and octet");
  const int i = threadIdx.x / (D / 2), m = threadIdx.x / O % 4, oct = threadIdx.x % O;
  if (i < heads) {
    uint32_t c[8], mask = 0;
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const int t = 16 * (y >> 2) + 4 * m + (y & 3);
      const bool in = t >= it.lo && t < it.hi;
      c[y] = in ? codes[i][t * LD + oct] : 0u;
      mask |= in ? 15u << (4 * y) : 0u;
    }
    transpose_nibbles(c);
    uint32_t* vc = reinterpret_cast<uint32_t*>(it.head + (long long)(it.h + i) * ph.bytes() + ph.vcode(it.row0)) +
                   (m * 16 + 8 * (oct & 1)) * (D / 16) + oct / 2;
    if (mask == 0xffffffffu) {
#pragma unroll
      for (int y = 0; y < 8; ++y) vc[y * (D / 16)] = c[y];
    } else if (mask) {
#pragma unroll
      for (int y = 0; y < 8; ++y) vc[y * (D / 16)] = (vc[y * (D / 16)] & ~mask) | c[y];
    }
  }
}

// The same blocks back; value codes through LDS, whose order is by channels.  Bound by HBM
// (272 to 278 us, 5.6 TB/s, for the cache above).
template <class T, int D>
__global__ __launch_bounds__(2 * D) void paged_read_kernel(const PagedRowsArgs a, const int hpw) {
  constexpr int TPT = D / 16;
  constexpr int G = D / 32;
  __shared__ uint32_t codes[16 * D / 8 * 2];
  const RowItem it = row_item<D>(a, hpw);
  const int tok = threadIdx.x / TPT, j = threadIdx.x % TPT;
  const bool on = tok >= it.lo && tok < it.hi;
  const PageHead<D> ph(a.log2_page);
  const int row = it.row0 + tok;
  T* dst = static_cast<T*>(const_cast<void*>(it.role == 0 ? a.k : a.v)) + rows_at(a, it, tok);
  const long long sh = it.role == 0 ? a.k_sh : a.v_sh;
  const int h_end = min(it.h + hpw, a.H);
  for (int h = it.h; h < h_end; ++h) {
    const uint8_t* head = it.head + (long long)h * ph.bytes();
    uint32_t c0 = 0, c1 = 0, w0 = 0, w1 = 0;
    if (it.head) {
      if (it.role == 1) {
        if (h > it.h) __syncthreads();
        const uint32_t* vc = reinterpret_cast<const uint32_t*>(head + ph.vcode(it.row0));
        codes[threadIdx.x] = vc[threadIdx.x];
        codes[threadIdx.x + 2 * D] = vc[threadIdx.x + 2 * D];
        __syncthreads();
      }
      if (on) {
        const uint32_t* words = reinterpret_cast<const uint32_t*>(head + ph.word(it.role, row));
        w0 = words[j >> 2];
        w1 = words[G / 2 + (j >> 2)];
        if (it.role == 0) {
          const uint32_t* kc = reinterpret_cast<const uint32_t*>(head + ph.kcode(row));
          c0 = kc[(j & 3) * G + (j >> 2)];
          c1 = kc[(j & 3) * G + G / 2 + (j >> 2)];
        } else {
          const int m = (tok >> 2) & 3, y = 4 * (tok >> 4) + (tok & 3);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int a0 = 8 * j + e, a1 = D / 2 + 8 * j + e;
            c0 |= ((codes[(m * 16 + a0 % 16) * (D / 16) + a0 / 16] >> (4 * y)) & 15) << (4 * e);
            c1 |= ((codes[(m * 16 + a1 % 16) * (D / 16) + a1 / 16] >> (4 * y)) & 15) << (4 * e);
          }
        }
      }
    }
    if (!on) continue;
    float x0[8], x1[8];
    const float s0 = __builtin_bit_cast(float, w0 & 0xffff0000u), o0 = __builtin_bit_cast(float, w0 << 16);
    const float s1 = __builtin_bit_cast(float, w1 & 0xffff0000u), o1 = __builtin_bit_cast(float, w1 << 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // (s * code is exact in fp32)
      x0[e] = fmaf(s0, (float)((c0 >> (4 * e)) & 15), o0);
      x1[e] = fmaf(s1, (float)((c1 >> (4 * e)) & 15), o1);
    }
    store8<T>(dst + h * sh + 8 * j, x0);
    store8<T>(dst + h * sh + D / 2 + 8 * j, x1);
  }
}

// ---------------------------------------------------------------------------
// Attention.  A workgroup takes 16 query rows of a group and a part of the
// tokens; its four waves deal the blocks of 32 tokens among them.  On
// v_mfma_f32_16x16x32_bf16, with m = lane / 16, S^T = K Q^T gives the lane its row
// lane % 16 and tokens 4 m + i of each half of the block (i: the result register),
// which is how the value codes lie: the lane's dword for channel block n holds
// channel 16 n + lane % 16 of those eight tokens.
// ---------------------------------------------------------------------------
constexpr int kPagedWaves = 4, kPagedRows = 16;

// Blocks of 32 tokens on their way through LDS: three stages a wave, filled by
// global-to-LDS loads two blocks ahead.
template <int D>
struct Stage {
  static constexpr int G = D / 32;
  static constexpr int V = 16 * D, W = 32 * D, BYTES = 32 * D + 1024;  // key codes; value codes; words
  static constexpr int LOADS = 2 * (D / 64) + 1;
  static constexpr int COUNT = 3;

  // The block of tokens row .. row + 32 of a page.
  FI static void fill(const uint8_t* head, const PageHead<D>& ph, int row, unsigned char* st, int lane) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
      __builtin_amdgcn_global_load_lds((const void*)(head + ph.kcode(row) + i * 1024 + lane * 16),
                                       (lds_void_t*)(st + i * 1024), 16, 0, 0);
    constexpr int CW = 2 * G;  // 16-byte pieces of 8 tokens' words
    const int wl = lane % (8 * CW);
    __builtin_amdgcn_global_load_lds(
        (const void*)(head + ph.word(wl / (4 * CW), row) + wl % (4 * CW) * 16), (lds_void_t*)(st + W), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
      __builtin_amdgcn_global_load_lds((const void*)(head + ph.vcode(row) + i * 1024 + lane * 16),
                                       (lds_void_t*)(st + V + i * 1024), 16, 0, 0);
  }
};

// What a lane reads of a stage.  The reads are written as instructions that the
// compiler does not see as LDS accesses: it cannot tell which load in flight fills
// which stage, and would wait for all of them.  They end with their own wait.
template <int D>
struct Block;
template <>
struct Block<128> {
  u32x4 k[2];  // key codes of token 16 u + lane % 16, octet lane / 16 of each group
  u32x4 v[2];  // value codes
  u32x4 w;     // words of token lane % 32: keys' in lanes below 32, values' above
  u32x4 wk[2]; // words of key token 16 u + lane % 16
  FI void read(uint32_t st, int lane) {
    const uint32_t ak = st + (lane & 15) * 64 + (lane >> 4) * 16, av = st + lane * 32;
    const uint32_t aw = st + lane * 16, ax = st + (lane & 15) * 16;
    asm volatile(
        "ds_read_b128 %0, %7\n\t"
        "ds_read_b128 %1, %7 offset:1024\n\t"
        "ds_read_b128 %2, %8 offset:2048\n\t"
        "ds_read_b128 %3, %8 offset:2064\n\t"
        "ds_read_b128 %4, %9 offset:4096\n\t"
        "ds_read_b128 %5, %10 offset:4096\n\t"
        "ds_read_b128 %6, %10 offset:4352\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(k[0]), "=&v"(k[1]), "=&v"(v[0]), "=&v"(v[1]), "=&v"(w), "=&v"(wk[0]), "=&v"(wk[1])
        : "v"(ak), "v"(av), "v"(aw), "v"(ax)
        : "memory");
  }
  FI uint32_t key(int u, int g) const { return k[u][g]; }
  FI uint32_t value(int n) const { return v[n / 4][n & 3]; }
};
template <>
struct Block<64> {
  u32x2 k[2];
  u32x4 v;
  u32x2 w, wk[2];
  FI void read(uint32_t st, int lane) {
    const uint32_t ak = st + (lane & 15) * 32 + (lane >> 4) * 8, av = st + lane * 16;
    const uint32_t aw = st + lane * 8, ax = st + (lane & 15) * 8;
    asm volatile(
        "ds_read_b64 %0, %6\n\t"
        "ds_read_b64 %1, %6 offset:512\n\t"
        "ds_read_b128 %2, %7 offset:1024\n\t"
        "ds_read_b64 %3, %8 offset:2048\n\t"
        "ds_read_b64 %4, %9 offset:2048\n\t"
        "ds_read_b64 %5, %9 offset:2176\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(k[0]), "=&v"(k[1]), "=&v"(v), "=&v"(w), "=&v"(wk[0]), "=&v"(wk[1])
        : "v"(ak), "v"(av), "v"(aw), "v"(ax)
        : "memory");
  }
  FI uint32_t key(int u, int g) const { return k[u][g]; }
  FI uint32_t value(int n) const { return v[n]; }
};

template <bool M>
struct Flag {
  static constexpr bool value = M;
};

// Four waves a workgroup, two workgroups a CU, blocks of the part dealt to the waves in
// turn, the next two blocks' 5 KB each in flight.  Per block a wave spends about 130
// instructions on taking codes out of dwords, 110 on scales and 60 on the softmax, beside
// 22 matrix instructions; that and HBM bound it together: 29K tokens of 40 heads on 8 of
// 128 (37 MB) in 16.6 us and 4.8 for the join, 16 sequences of 4 to 8K tokens (64 MB) in
// 23.0 and 4.0.  One query token over 200 takes 7.6 us, most of it a few loads that need
// each other (arguments, page, block).
// Measured and dropped: the next block in registers instead of LDS (17.0 us against 16.3,
// 25.5 against 22.4 for the 16 sequences); two tiles of 16 rows a workgroup, which read the
// codes once for both but leave one workgroup a CU (32 rows over 29K tokens 38.2 us against
// 24.6, 256 rows 174 against 125; d_h 64 within 6% either way); eight waves and one workgroup
// a CU (29K tokens 17.1 against 16.8 us, 64 sequences of 1,000 29.8 against 24.2, though 32 of
// 1.5 to 3K 30.5 against 33.8); parts for 256, 384 or 1,024
// workgroups instead of 512 (18.4, 17.8 and 19.5 us against 16.7).
//
// The keys' offsets cost a matrix instruction a tile: the words of a token, as they
// are stored, are eight bf16 numbers (o_g, s_g), and the other operand holds
// sum(q_g) and what takes the operands' 16 out again, -16 sum(q_g), each split into
// three bf16 terms (24 bits) over three of its four octets.
template <int D, bool F32>
__global__ __launch_bounds__(kPagedWaves * 64, 2) void paged_attention_kernel(const PagedAttnArgs a) {
  constexpr int G = D / 32, NC = D / 16, S = F32 ? 3 : 1, R = kPagedRows;
  constexpr int NW = kPagedWaves;
  typedef Stage<D> St;
  constexpr int WB = 64 * G * 2;  // floats a wave: scales and offsets [role][G][32]
  constexpr int STAGED = NW * (St::COUNT * St::BYTES), JOINED = NW * D * R * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char stages[STAGED > JOINED ? STAGED : JOINED];
  __shared__ __attribute__((aligned(16))) float lds[NW * WB];
  __shared__ float sm[NW][R], sl[NW][R];

  const int lane = threadIdx.x & 63, col = lane & 15, m4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AttnSeqs& s = a.s;
  const AttnItem it = attn_item(s, R);
  const int t = it.t, n_rows = it.rows;
  const int row0 = it.tile * R;
  const float c = a.io.c;
  float* sc = lds + wave * WB;
  float* of = sc + 64 * G;
  unsigned char* my_stages = stages + wave * (St::COUNT * St::BYTES);

  const int first_last = last_key(s, it, divide(min(row0, n_rows - 1), s.by_g));
  const int end_last = last_key(s, it, divide(min(row0 + R - 1, n_rows - 1), s.by_g));
  const int lo = it.part * s.chunk;
  const int hi = min(end_last + 1, it.parts == 1 ? t : min(t, lo + s.chunk));
  const int P = 1 << a.log2_page;
  const PageHead<D> ph(a.log2_page);
  const int32_t* table = a.table + it.b * a.table_stride;
  const long long head_at = (long long)it.h * ph.bytes();

  // The wave's blocks: i = 0, 1, .. at tokens first + i * 32 NW.  Lane i holds the page
  // of block i of each 64.
  const int first = lo + 32 * wave;
  const int n_blocks = first < hi ? (hi - first + 32 * NW - 1) / (32 * NW) : 0;
  auto pages_from = [&](int i) {
    const int at = first + (i + lane) * 32 * NW;
    return at < hi ? table[at >> a.log2_page] : -1;
  };
  int pages = -1;
  auto page_of = [&](int i) { return __builtin_amdgcn_readlane(pages, i & 63); };
  int held = 0;  // bit s: stage s holds a block of a page, not of a hole
  // Block i to stage i % 3 (a hole's, too: it loads from page 0 and is masked).
  auto fill = [&](int i, int st) {
    if (i >= n_blocks) return;
    if ((i & 63) == 0) {
      pages = pages_from(i);
      asm volatile("" : "+v"(pages));  // (waited for here, not at every block's fill)
    }
    const int page = page_of(i);
    const bool in = (unsigned)page < (unsigned)a.n_pages;
    held = (held & ~(1 << st)) | ((int)in << st);
    const uint8_t* head = a.pages + (long long)(in ? page : 0) * a.page_bytes + head_at;
    St::fill(head, ph, (first + i * 32 * NW) & (P - 1), my_stages + st * St::BYTES, lane);
  };
  // the queries and the first block on their way before either is used
  typedef uint32_t QRaw[F32 ? 8 : 4];
  QRaw raw_q[G];
  const int r = min(row0 + col, n_rows - 1);
  const int token = divide(r, s.by_g), head = it.h * s.G + r - token * s.G;
  const int last = last_key(s, it, token);
  const uint8_t* row = static_cast<const uint8_t*>(a.io.q) +
                       (seq_at(it.b, it.row0, a.io.q_sb, a.io.q_st) + token * a.io.q_st + head * a.io.q_sh) *
                           (F32 ? 4 : 2);
#pragma unroll
  for (int y = 0; y < G; ++y) load_dwords<F32 ? 8 : 4>(row + (32 * y + 8 * m4) * (F32 ? 4 : 2), raw_q[y]);
  fill(0, 0);
  fill(1, 1);

  bf16x8 q[S][G];
  bf16x8 qo = {};  // against the words
#pragma unroll
  for (int y = 0; y < G; ++y) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = raw_q[y][F32 ? e : e / 2];
      const float f = __builtin_bit_cast(float, F32 ? w : e & 1 ? w & 0xffff0000u : w << 16);
      sum += f;
      float p[S];
      split<S>(f, p);
#pragma unroll
      for (int z = 0; z < S; ++z) q[z][y][e < 4 ? 2 * e : 2 * (e - 4) + 1] = (__bf16)p[z];
    }
    sum = add_xor32(add_xor16(sum));
    float p[3];
    split<3>(sum, p);
    const float mine = m4 == 0 ? p[0] : m4 == 1 ? p[1] : m4 == 2 ? p[2] : 0.0f;
    qo[2 * y] = (__bf16)mine;
    qo[2 * y + 1] = (__bf16)(mine * (F32 ? 8.0f : -16.0f));
  }

  const Codes codes;
  f32x4 o[NC] = {};    // sum of (p s) times the operand: row col, channels 16 n + 4 m4 + i
  f32x4 ps[G] = {};    // sum of the rounded p s
  float po[G] = {};    // sum of p times the offset, over the lane's tokens
  float m = kNoMax, l = 0.0f;
  float cr = c;        // the unit of m

  // masked: some row of the tile does not see all of the block's tokens, or it is a hole
  auto block = [&](auto masked, const Block<D>& x, int t0, bool in) {
    constexpr bool M = decltype(masked)::value;
    // scales, and the values' offsets moved to code 8, to the lanes that need them.  Words
    // of tokens that no row sees count as 0, so that nothing below meets a NaN of theirs.
    const bool live = !M || (in && t0 + (lane & 31) < hi);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int y = 0; y < G; ++y) {
      const uint32_t w = live ? x.w[y] : 0u;
      const float f = __builtin_bit_cast(float, w & 0xffff0000u);
      sc[(lane >> 5) * 32 * G + 32 * y + (lane & 31)] = f;
      of[(lane >> 5) * 32 * G + 32 * y + (lane & 31)] = fmaf(f, 8.0f, __builtin_bit_cast(float, w << 16));
    }
    __builtin_amdgcn_wave_barrier();

    float p[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      union {
        uint32_t d[4];
        bf16x8 v;
      } wk = {{0, 0, 0, 0}};
#pragma unroll
      for (int y = 0; y < G; ++y) wk.d[y] = x.wk[u][y];
      f32x4 v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wk.v, qo, f32x4{}, 0, 0, 0);
#pragma unroll
      for (int y = 0; y < G; ++y) {
        const bf16x8 kc = codes.operand<F32>(x.key(u, y));
        const f32x4 ks = *reinterpret_cast<const f32x4*>(sc + 32 * y + 16 * u + 4 * m4);
        f32x4 d = {};
#pragma unroll
        for (int z = 0; z < S; ++z)
          d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kc, q[z][y], d, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(ks[i], d[i], v[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[4 * u + i] = v[i];
    }
    if (M) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = t0 + 16 * (i >> 2) + 4 * m4 + (i & 3);
        if (!in || k > last || k >= hi) p[i] = -INFINITY;
      }
    }
    float mx = p[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, p[i]);
    const float top = max_xor32(max_xor16(mx));
    mx = top * cr;
    if (__any(mx > m + kRaise)) {
      const float nm = mx > m + kRaise ? mx : m;  // (each row by its own scores alone)
      float f = __builtin_amdgcn_exp2f(m - nm);
      if (__any(far_max(nm) || cr != c))
        f = raise(top, c, true, cr, m);
      else
        m = nm;
      l *= f;
#pragma unroll
      for (int y = 0; y < NC; ++y) o[y] *= f;
#pragma unroll
      for (int y = 0; y < G; ++y) {
        if (!F32) ps[y] *= f;
        po[y] *= f;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], cr, -m));
      l += p[i];
    }

    const bf16x8 one = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f,
                        (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int y = 0; y < G; ++y) {
      const bf16x8 v0 = codes.operand<F32>(x.value(2 * y)), v1 = codes.operand<F32>(x.value(2 * y + 1));
      f32x4 zs[2], zo[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        zs[u] = *reinterpret_cast<const f32x4*>(sc + 32 * G + 32 * y + 16 * u + 4 * m4);
        zo[u] = *reinterpret_cast<const f32x4*>(of + 32 * G + 32 * y + 16 * u + 4 * m4);
      }
      float f[8], sum = po[y];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = p[i] * zs[i >> 2][i & 3];
        if (M) {
          // what a row does not see has weight 0, and may be NaN
          const bool seen = t0 + 16 * (i >> 2) + 4 * m4 + (i & 3) <= last;
          f[i] = seen ? f[i] : 0.0f;
          sum = seen ? fmaf(p[i], zo[i >> 2][i & 3], sum) : sum;
        } else {
          sum = fmaf(p[i], zo[i >> 2][i & 3], sum);
        }
      }
      po[y] = sum;
      float w[8][S];
#pragma unroll
      for (int i = 0; i < 8; ++i) split<S>(f[i], w[i]);
#pragma unroll
      for (int z = 0; z < S; ++z) {
        union {
          uint32_t u[4];
          bf16x8 v;
        } pw;
#pragma unroll
        for (int i = 0; i < 4; ++i) pw.u[i] = pack_bf16(w[i][z], w[4 + i][z]);
        if (!F32) ps[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, pw.v, ps[y], 0, 0, 0);
        o[2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pw.v, o[2 * y], 0, 0, 0);
        o[2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pw.v, o[2 * y + 1], 0, 0, 0);
      }
    }
  };
  auto turn = [&](int i, int st, int later) {
    if (i >= n_blocks) return;
    fill(i + 2, later);
    // at most the loads of the blocks after this one are outstanding
    const int after = min(n_blocks - 1 - i, 2);
    if (after == 2)
      __builtin_amdgcn_s_waitcnt(wait_vm_only(2 * St::LOADS));
    else if (after == 1)
      __builtin_amdgcn_s_waitcnt(wait_vm_only(St::LOADS));
    else
      __builtin_amdgcn_s_waitcnt(wait_vm_only(0));
    Block<D> x;
    x.read(lds_addr(my_stages + st * St::BYTES), lane);
    const int t0 = first + i * 32 * NW;
    const bool in = (held >> st) & 1;
    if (!in || t0 + 31 > first_last || t0 + 32 > hi)
      block(Flag<true>(), x, t0, in);
    else
      block(Flag<false>(), x, t0, true);
  };
  int st = 0;
  for (int i = 0; i < n_blocks; ++i) {
    const int later = st == 0 ? 2 : st - 1;  // (i + 2) % 3
    turn(i, st, later);
    st = st == 2 ? 0 : st + 1;
  }

  // the lane's rows: out of the codes' 16 (with the 8 of the moved offsets), the
  // offsets of all lanes' tokens
  l = add_xor32(add_xor16(l));
  if (__any(far_max(m))) {  // (rare: whether the row saw a key, by the wave's first token in a page)
    unsigned long long in = 0;
    int i = 0;
    for (; i < n_blocks && !in; i += 64) in = __ballot((unsigned)pages_from(i) < (unsigned)a.n_pages);
    m = end_max(m, cr, c, l, in && first + (i - 64 + __builtin_ctzll(in)) * 32 * NW <= last);
  }
#pragma unroll
  for (int y = 0; y < G; ++y) {
    const float x = add_xor32(add_xor16(po[y]));
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[2 * y + z][i] += F32 ? x : fmaf(-24.0f, ps[y][i], x);
  }
  if (m4 == 0) {
    sm[wave][col] = m;
    sl[wave][col] = l;
  }
  __syncthreads();
  f32x4* sums = reinterpret_cast<f32x4*>(stages);
  float mm = kNoMax;
#pragma unroll
  for (int x = 0; x < NW; ++x) mm = fmaxf(mm, sm[x][col]);
  const float f = __builtin_amdgcn_exp2f(m - mm);
#pragma unroll
  for (int y = 0; y < NC; ++y) sums[sum_slot<R, D>(wave, col, 4 * y + m4)] = o[y] * f;
  __syncthreads();
  write_joined<R, D, NW, F32>(a.io, s, it, row0, sums, sm, sl);
}

template <int D>
hipError_t launch(int dtype, const PagedAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.s.n_items * a.s.H));
  const int threads = kPagedWaves * 64;
  if (dtype == HF_F32)
    paged_attention_kernel<D, true><<<grid, threads, 0, st>>>(a);
  else
    paged_attention_kernel<D, false><<<grid, threads, 0, st>>>(a);
  return hipGetLastError();
}

// Heads a workgroup, one or four: four where there are so many blocks that one launch's
// workgroups come and go many times, and where a block's angles are worth sharing.
// Measured with one and with four, us, rows of 8 heads of 128 in bf16, append and read:
// 10 layers of 7,282 tokens 94 + 69 and 100 + 67, 20 layers 204 + 152 and 178 + 134,
// 40 layers 408 + 308 and 363 + 283; rotated, one layer of 2,000 tokens 7.5 and 8.0, of
// 8,000 18.9 and 16.4, of 30,000 64 and 46.
int heads_per_workgroup(const PagedRowsArgs& a) {
  const int64_t heads = (int64_t)a.n_blocks * a.n_layers * a.H;
  return heads >= (a.rotate ? 1024 : 32768) ? kHeads : 1;
}

template <class T, int D>
void append(dim3 grid, const PagedRowsArgs& a, int hpw, hipStream_t s) {
  if (a.rotate)
    paged_append_kernel<T, D, true><<<grid, 2 * D, 0, s>>>(a, hpw);
  else
    paged_append_kernel<T, D, false><<<grid, 2 * D, 0, s>>>(a, hpw);
}

}  // namespace

// Times as the rule weighs them, with two workgroups a CU, parts of 128 to 7,296 tokens; now,
// from L2, us of start and ns a key: bf16 of 128 6.4 + 14.1, of 64 4.7 + 8.6; fp32 8.4 + 29.1
// and 5.6 + 16.3.
AttnShape paged_shape(int dtype, int d_h) {
  AttnShape sh;
  const bool f32 = dtype == HF_F32, wide = d_h == 128;
  sh.rows = kPagedRows;
  sh.by_keys = 1;
  sh.resident = 1;
  sh.wg_target = 512;
  sh.step = 32 * kPagedWaves;
  sh.ns_start = f32 ? (wide ? 10000 : 3000) : wide ? 6000 : 4800;
  sh.ns_key = f32 ? (wide ? 33 : 21) : wide ? 16 : 11;
  return sh;
}

hipError_t launch_paged_attention(int dtype, int d_h, const PagedAttnArgs& a, hipStream_t s) {
  return d_h == 128 ? launch<128>(dtype, a, s) : launch<64>(dtype, a, s);
}

hipError_t launch_paged_append(int dtype, int d_h, const PagedRowsArgs& a0, hipStream_t s) {
  PagedRowsArgs a = a0;
  const int hpw = heads_per_workgroup(a);
  a.by_groups = make_divide((a.H + hpw - 1) / hpw);
  const dim3 grid((unsigned)(a.n_blocks * ((a.H + hpw - 1) / hpw)), 2, (unsigned)a.n_layers);
  if (dtype == HF_BF16)
    d_h == 128 ? append<uint16_t, 128>(grid, a, hpw, s) : append<uint16_t, 64>(grid, a, hpw, s);
  else
    d_h == 128 ? append<float, 128>(grid, a, hpw, s) : append<float, 64>(grid, a, hpw, s);
  return hipGetLastError();
}

hipError_t launch_paged_read(int dtype, int d_h, const PagedRowsArgs& a0, hipStream_t s) {
  PagedRowsArgs a = a0;
  const int hpw = heads_per_workgroup(a);
  a.by_groups = make_divide((a.H + hpw - 1) / hpw);
  const dim3 grid((unsigned)(a.n_blocks * ((a.H + hpw - 1) / hpw)), 2, (unsigned)a.n_layers);
  if (dtype == HF_BF16) {
    if (d_h == 128) paged_read_kernel<uint16_t, 128><<<grid, 256, 0, s>>>(a, hpw);
    else paged_read_kernel<uint16_t, 64><<<grid, 128, 0, s>>>(a, hpw);
  } else {
    if (d_h == 128) paged_read_kernel<float, 128><<<grid, 256, 0, s>>>(a, hpw);
    else paged_read_kernel<float, 64><<<grid, 128, 0, s>>>(a, hpw);
  }
  return hipGetLastError();
}

}  // namespace hf
