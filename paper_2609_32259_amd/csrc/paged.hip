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

namespace hf {
namespace {

// ---------------------------------------------------------------------------
// Rows in and out.  A workgroup takes a block of 32 tokens (the unit of the value
// codes' order) of one sequence, layer, role and head; 16 channels a thread.
// ---------------------------------------------------------------------------

struct RowItem {
  int b, l, h, role;
  int tok0;          // first token of the block
  int lo, hi;        // tokens of the call in it, relative to tok0
  uint8_t* head;     // the head's part of the page, or nullptr (a hole)
  int row0;          // the block's first row in the page
};

template <int D>
FI RowItem row_item(const PagedRowsArgs& a, int hpw) {
  RowItem it;
  int i = blockIdx.x;
  const int groups = (a.H + hpw - 1) / hpw;
  it.h = (i % groups) * hpw;
  i /= groups;
  it.role = blockIdx.y;
  it.l = blockIdx.z;
  const int b = find_seq(a.blk0, a.B, i);
  it.b = b;
  const int blk = a.start[b] / 32 + (i - a.blk0[b]);
  it.tok0 = blk * 32;
  it.lo = max(a.start[b] - it.tok0, 0);
  it.hi = min(a.start[b] + a.n[b] - it.tok0, 32);
  const int page = a.table[b * a.table_stride + (it.tok0 >> a.log2_page)];
  it.row0 = it.tok0 & ((1 << a.log2_page) - 1);
  it.head = nullptr;
  if ((unsigned)page < (unsigned)a.n_pages)
    it.head = a.pages + ((long long)it.l * a.n_pages + page) * a.page_bytes;
  return it;
}

// Offsets in a head's part of a page.
template <int D>
struct PageHead {
  static constexpr int G = D / 32;
  int P;
  FI PageHead(int log2_page) : P(1 << log2_page) {}
  FI int bytes() const { return P * (D + 8 * G); }
  FI int kcode(int row) const { return row * (D / 2); }
  FI int vcode(int row) const { return P * (D / 2) + row * (D / 2); }  // row: of a block's first token
  FI int word(int role, int row) const { return P * D + (role * P + row) * (4 * G); }
};

template <class T>
FI void load8(const T* p, float (&x)[8]);
template <>
FI void load8<uint16_t>(const uint16_t* p, float (&x)[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, v[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
  }
}
template <>
FI void load8<float>(const float* p, float (&x)[8]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}

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

FI float bf16_round(float x) { return (float)(__bf16)x; }

// Codes and word of a group spread over four lanes (l, l ^ 1, l ^ 2, l ^ 3), eight
// channels a lane.  Codes as a dword, channel j at nibble j.
FI uint32_t code_group(const float (&x)[8], uint32_t& word) {
#pragma clang fp contract(off)
  float lo = x[0], hi = x[0];
  bool nan = x[0] != x[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) {
    lo = fminf(lo, x[j]);
    hi = fmaxf(hi, x[j]);
    nan = nan || x[j] != x[j];
  }
  // (fminf and fmaxf pass NaN by)
  lo = nan ? NAN : lo;
#pragma unroll
  for (int m = 1; m <= 2; m <<= 1) {
    const float ol = __shfl_xor(lo, m), oh = __shfl_xor(hi, m);
    lo = lo != lo || ol != ol ? NAN : fminf(lo, ol);
    hi = fmaxf(hi, oh);
  }
  const float o = bf16_round(lo);
  float s = bf16_round((hi - lo) / 15.0f);
  if (!finite_bits(o) || !finite_bits(s)) {
    word = 0x7fc07fc0u;  // NaN, NaN
    return 0;
  }
  if (s < 0x1p-100f) s = 0.0f;
  word = __builtin_bit_cast(uint32_t, s) | (__builtin_bit_cast(uint32_t, o) >> 16);
  uint32_t c = 0;
  const float d = s > 0.0f ? s : INFINITY;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // a true quotient: what lies halfway between two codes goes to the even one
    const float q = fminf(fmaxf(rintf((x[j] - o) / d), 0.0f), 15.0f);
    c |= (uint32_t)(int)q << (4 * j);
  }
  return c;
}

// cos and sin of pos * w_k for the block's 32 positions, to LDS [32][D/2], fp64
// angles rounded once.  Four chains a channel pair, eight positions each: one sine
// and cosine at the chain's first position, then a complex product with the step's
// (error 8 * 2^-53).  A block with up to four tokens computes just theirs.
template <int D>
FI void fill_angles(const PagedRowsArgs& a, const RowItem& it, float2* cs) {
  constexpr int HD = D / 2;
  const int k = threadIdx.x % HD, m = threadIdx.x / HD;  // m < 4
  const double w = a.w[k];
  const double base = (double)a.pos0[it.b] + it.tok0;
  double c, s;
  if (it.hi - it.lo <= 4) {
    const int j = it.lo + m;
    if (j < it.hi) {
      sincos((base + j) * w, &s, &c);
      cs[j * HD + k] = make_float2((float)c, (float)s);
    }
    return;
  }
  double dc, ds;
  sincos(w, &ds, &dc);
  sincos((base + 8 * m) * w, &s, &c);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cs[(8 * m + j) * HD + k] = make_float2((float)c, (float)s);
    const double t = c * dc - s * ds;
    s = s * dc + c * ds;
    c = t;
  }
}

template <class T, int D>
__global__ __launch_bounds__(2 * D) void paged_append_kernel(const PagedRowsArgs a, const int hpw) {
  constexpr int TPT = D / 16;  // threads a token
  constexpr int G = D / 32;
  __shared__ float2 cs[32 * D / 2];
  __shared__ uint32_t codes[32 * D / 8];  // [token][channel] nibbles
  const RowItem it = row_item<D>(a, hpw);
  if (!it.head) return;
  const int tok = threadIdx.x / TPT, j = threadIdx.x % TPT;
  const bool on = tok >= it.lo && tok < it.hi;
  const bool rot = a.rotate && it.role == 0;
  if (rot) {
    fill_angles<D>(a, it, cs);
    __syncthreads();
  }
  const PageHead<D> ph(a.log2_page);
  const int row = it.row0 + tok;
  const T* src = it.role == 0
                     ? static_cast<const T*>(a.k) + a.k_off[it.b] + it.l * a.k_sl +
                           (long long)(it.tok0 + tok - a.start[it.b]) * a.k_st
                     : static_cast<const T*>(a.v) + a.v_off[it.b] + it.l * a.v_sl +
                           (long long)(it.tok0 + tok - a.start[it.b]) * a.v_st;
  const long long sh = it.role == 0 ? a.k_sh : a.v_sh;
  const int h_end = min(it.h + hpw, a.H);
  for (int h = it.h; h < h_end; ++h) {
    uint8_t* head = it.head + (long long)h * ph.bytes();
    uint32_t c0 = 0, c1 = 0, w0 = 0, w1 = 0;
    if (on) {  // (a group's four lanes hold the same token)
      float x0[8], x1[8];  // channels 8 j .. and D/2 + 8 j ..: rotation pairs
      load8<T>(src + h * sh + 8 * j, x0);
      load8<T>(src + h * sh + D / 2 + 8 * j, x1);
      if (rot) {
#pragma clang fp contract(off)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 r = cs[tok * (D / 2) + 8 * j + e];
          const float u = x0[e], v = x1[e];
          x0[e] = u * r.x - v * r.y;
          x1[e] = v * r.x + u * r.y;
        }
      }
      c0 = code_group(x0, w0);
      c1 = code_group(x1, w1);
      uint32_t* words = reinterpret_cast<uint32_t*>(head + ph.word(it.role, row));
      if ((j & 3) == 0) {
        words[j >> 2] = w0;
        words[G / 2 + (j >> 2)] = w1;
      }
      if (it.role == 0) {
        uint32_t* kc = reinterpret_cast<uint32_t*>(head + ph.kcode(row));
        kc[(j & 3) * G + (j >> 2)] = c0;
        kc[(j & 3) * G + G / 2 + (j >> 2)] = c1;
      }
    }
    if (it.role == 0) continue;
    // Value codes: to the order of the block, through LDS.
    codes[tok * (D / 8) + j] = c0;
    codes[tok * (D / 8) + D / 16 + j] = c1;
    __syncthreads();
    const uint8_t* cb = reinterpret_cast<const uint8_t*>(codes);
    uint32_t* vc = reinterpret_cast<uint32_t*>(head + ph.vcode(it.row0));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = threadIdx.x + i * 2 * D;  // dword of the block
      const int n = at % (D / 16), c = at / (D / 16) % 16, m = at / D;
      const int ch = 16 * n + c;
      uint32_t x = 0, mask = 0;
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int t = 16 * (y >> 2) + 4 * m + (y & 3);
        const uint32_t nib = (cb[t * (D / 2) + ch / 2] >> (4 * (ch & 1))) & 15;
        if (t >= it.lo && t < it.hi) {
          x |= nib << (4 * y);
          mask |= 15u << (4 * y);
        }
      }
      if (mask == 0xffffffffu)
        vc[at] = x;
      else if (mask)
        vc[at] = (vc[at] & ~mask) | x;
    }
    if (h + 1 < h_end) __syncthreads();
  }
}

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
  T* dst = it.role == 0 ? static_cast<T*>(const_cast<void*>(a.k)) + a.k_off[it.b] + it.l * a.k_sl +
                              (long long)(it.tok0 + tok - a.start[it.b]) * a.k_st
                        : static_cast<T*>(const_cast<void*>(a.v)) + a.v_off[it.b] + it.l * a.v_sl +
                              (long long)(it.tok0 + tok - a.start[it.b]) * a.v_st;
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
// Attention.  A workgroup takes 16 NT query rows of a group and a part of the
// tokens; its four waves deal the blocks of 32 tokens among them.  On
// v_mfma_f32_16x16x32_bf16, with m = lane / 16, S^T = K Q^T gives the lane its row
// lane % 16 and tokens 4 m + i of each half of the block (i: the result register),
// which is how the value codes lie: the lane's dword for channel block n holds
// channel 16 n + lane % 16 of those eight tokens.
// ---------------------------------------------------------------------------
constexpr int kPagedWaves = 4;

// Two codes of a dword, nibbles n and n + 4, as bf16 16 + code.
FI uint32_t two_codes(uint32_t w, int n) {
  // the code to bits 3..6 of each half, under the exponent of 16
  const uint32_t x = n == 0 ? w << 3 : w >> (4 * n - 3);
  return (x & 0x00780078u) | 0x41804180u;
}
FI bf16x8 eight_codes(uint32_t w) {
  union {
    uint32_t u[4];
    bf16x8 v;
  } x;
#pragma unroll
  for (int n = 0; n < 4; ++n) x.u[n] = two_codes(w, n);
  return x.v;
}

// The same as code - 8, for fp32: 16 + code beside sums of up to 16 would cost four
// more bits of the fp32 accumulation than code - 8 does.
FI bf16x8 eight_centred(uint32_t w) {
  union {
    uint32_t u[4];
    bf16x8 v;
  } x;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const uint32_t p = two_codes(w, n);
    const float lo = __builtin_bit_cast(float, p << 16) - 24.0f;
    const float hi = __builtin_bit_cast(float, p & 0xffff0000u) - 24.0f;
    x.u[n] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo),
                                   0x07060302u);  // (exact: the upper halves)
  }
  return x.v;
}
template <bool F32>
FI bf16x8 code_operand(uint32_t w) {
  return F32 ? eight_centred(w) : eight_codes(w);
}

// x as S bf16 terms whose sum holds 8 S bits of it.
template <int S>
FI void split(float x, float (&t)[S]) {
#pragma unroll
  for (int i = 0; i < S; ++i) {
    t[i] = bf16_round(x);
    x -= t[i];
  }
}

// What a lane holds of a block of 32 tokens, as it is loaded.
template <int D>
struct Block {
  static constexpr int G = D / 32;
  uint32_t k[2][G];    // key codes of token 16 u + lane % 16, octet lane / 16 of each group
  uint32_t v[D / 16];  // value codes
  uint32_t w[G];       // words of token lane % 32: keys' in lanes below 32, values' above
  int page;
};

template <int N>
FI void load_dwords(const uint8_t* p, uint32_t (&x)[N]) {
  if (N == 2) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    x[0] = v[0];
    x[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i + e] = v[e];
    }
  }
}

template <bool M>
struct Flag {
  static constexpr bool value = M;
};

// Four waves a workgroup (two workgroups a CU with up to 16 rows), blocks of the part
// dealt to them in turn, the next block's 5 KB in flight.  Per block a wave spends
// about 130 instructions on taking codes out of dwords, 110 on scales and 60 on the
// softmax, beside 22 matrix instructions.
//
// The keys' offsets cost a matrix instruction a tile: the words of a token, as they
// are stored, are eight bf16 numbers (o_g, s_g), and the other operand holds
// sum(q_g) and what takes the operands' 16 out again, -16 sum(q_g), each split into
// three bf16 terms (24 bits) over three of its four octets.
template <int D, int NT, bool F32>
__global__ __launch_bounds__(kPagedWaves * 64, NT == 1 ? 2 : 1) void paged_attention_kernel(
    const PagedAttnArgs a) {
  constexpr int G = D / 32, NC = D / 16, S = F32 ? 3 : 1, R = 16 * NT;
  constexpr int NW = kPagedWaves;
  constexpr int WB = 64 * G * 3;  // floats a wave: scales and offsets [role][G][32], words [64][G]
  __shared__ __attribute__((aligned(16))) float lds[WB > D * R ? NW * WB : NW * D * R];
  __shared__ float sm[NW][R], sl[NW][R];
  typedef uint32_t uG __attribute__((ext_vector_type(G)));

  const int lane = threadIdx.x & 63, col = lane & 15, m4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AttnSeqs& s = a.s;
  const AttnItem it = attn_item(s, R);
  const int b = it.b, t = s.t[b];
  const int n_rows = s.n[b] * s.G;
  const int row0 = it.tile * R;
  const float c = a.io.c;
  float* sc = lds + wave * WB;
  float* of = sc + 64 * G;
  uG* words = reinterpret_cast<uG*>(of + 64 * G);

  const int first_last = last_key(s, b, min(row0, n_rows - 1) / s.G);
  const int end_last = last_key(s, b, min(row0 + R - 1, n_rows - 1) / s.G);
  const int lo = it.part * s.chunk;
  const int hi = min(end_last + 1, s.parts[b] == 1 ? t : min(t, lo + s.chunk));
  const int P = 1 << a.log2_page;
  const PageHead<D> ph(a.log2_page);
  const int32_t* table = a.table + b * a.table_stride;
  const long long head_at = (long long)it.h * ph.bytes();

  // Block at token t0 (a hole's, too: it loads from page 0 and is masked).
  auto page_of = [&](int t0) { return t0 < hi ? table[t0 >> a.log2_page] : -1; };
  auto load = [&](Block<D>& x, int t0, int page) {
    x.page = page;
    if (t0 >= hi) return;
    const bool in = (unsigned)page < (unsigned)a.n_pages;
    const uint8_t* head = a.pages + (long long)(in ? page : 0) * a.page_bytes + head_at;
    const int row = t0 & (P - 1);
    load_dwords<G>(head + ph.kcode(row) + (col * (D / 2) + m4 * 4 * G), x.k[0]);
    load_dwords<G>(head + ph.kcode(row + 16) + (col * (D / 2) + m4 * 4 * G), x.k[1]);
    load_dwords<G>(head + ph.word(lane >> 5, row + (lane & 31)), x.w);
    load_dwords<NC>(head + ph.vcode(row) + lane * 4 * NC, x.v);
  };
  // the queries and the first block on their way before either is used
  typedef uint32_t QRaw[F32 ? 8 : 4];
  QRaw raw_q[NT][G];
  int last[NT];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    const int r = min(row0 + 16 * x + col, n_rows - 1);
    const int token = r / s.G, g = r - token * s.G;
    last[x] = last_key(s, b, token);
    const long long at = s.q_off[b] + (long long)token * a.io.q_st + (long long)(it.h * s.G + g) * a.io.q_sh;
    const uint8_t* row = static_cast<const uint8_t*>(a.io.q) + at * (F32 ? 4 : 2);
#pragma unroll
    for (int y = 0; y < G; ++y) load_dwords<F32 ? 8 : 4>(row + (32 * y + 8 * m4) * (F32 ? 4 : 2), raw_q[x][y]);
  }
  Block<D> x0, x1;
  int t0 = lo + 32 * wave;
  const int page0 = page_of(t0);
  int next_page = page_of(t0 + 32 * NW);
  load(x0, t0, page0);

  bf16x8 q[NT][S][G];
  bf16x8 qo[NT];   // against the words
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    qo[x] = bf16x8{};
#pragma unroll
    for (int y = 0; y < G; ++y) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = raw_q[x][y][F32 ? e : e / 2];
        const float f = __builtin_bit_cast(float, F32 ? w : e & 1 ? w & 0xffff0000u : w << 16);
        sum += f;
        float p[S];
        split<S>(f, p);
#pragma unroll
        for (int z = 0; z < S; ++z) q[x][z][y][e < 4 ? 2 * e : 2 * (e - 4) + 1] = (__bf16)p[z];
      }
      sum = add_xor32(add_xor16(sum));
      float p[3];
      split<3>(sum, p);
      const float mine = m4 == 0 ? p[0] : m4 == 1 ? p[1] : m4 == 2 ? p[2] : 0.0f;
      qo[x][2 * y] = (__bf16)mine;
      qo[x][2 * y + 1] = (__bf16)(mine * (F32 ? 8.0f : -16.0f));
    }
  }

  f32x4 o[NT][NC] = {};    // sum of (p s) times the operand: row col, channels 16 n + 4 m4 + i
  f32x4 ps[NT][G] = {};    // sum of the rounded p s
  float po[NT][G] = {};    // sum of p times the offset, over the lane's tokens
  float m[NT], l[NT];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    m[x] = kNoMax;
    l[x] = 0.0f;
  }

  // masked: some row of the tile does not see all of the block's tokens, or it is a hole
  auto block = [&](auto masked, const Block<D>& x, int t0, bool in) {
    constexpr bool M = decltype(masked)::value;
    // scales, and the values' offsets moved to code 8, to the lanes that need them.  Words
    // of tokens that no row sees count as 0, so that nothing below meets a NaN of theirs.
    const bool live = !M || (in && t0 + (lane & 31) < hi);
    uG raw;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int y = 0; y < G; ++y) {
      const uint32_t w = live ? x.w[y] : 0u;
      raw[y] = w;
      const float f = __builtin_bit_cast(float, w & 0xffff0000u);
      sc[(lane >> 5) * 32 * G + 32 * y + (lane & 31)] = f;
      of[(lane >> 5) * 32 * G + 32 * y + (lane & 31)] = fmaf(f, 8.0f, __builtin_bit_cast(float, w << 16));
    }
    words[lane] = raw;
    __builtin_amdgcn_wave_barrier();

    float p[NT][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      union {
        uint32_t d[4];
        bf16x8 v;
      } wk = {{0, 0, 0, 0}};
      const uG w = words[16 * u + col];
#pragma unroll
      for (int y = 0; y < G; ++y) wk.d[y] = w[y];
      f32x4 v[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
        v[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wk.v, qo[n], f32x4{}, 0, 0, 0);
#pragma unroll
      for (int y = 0; y < G; ++y) {
        const bf16x8 kc = code_operand<F32>(x.k[u][y]);
        const f32x4 ks = *reinterpret_cast<const f32x4*>(sc + 32 * y + 16 * u + 4 * m4);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          f32x4 d = {};
#pragma unroll
          for (int z = 0; z < S; ++z)
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kc, q[n][z][y], d, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[n][i] = fmaf(ks[i], d[i], v[n][i]);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[n][4 * u + i] = v[n][i];
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (M) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = t0 + 16 * (i >> 2) + 4 * m4 + (i & 3);
          if (!in || k > last[n] || k >= hi) p[n][i] = -INFINITY;
        }
      }
      float mx = p[n][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, p[n][i]);
      mx = max_xor32(max_xor16(mx)) * c;
      if (__any(mx > m[n] + kRaise)) {
        const float nm = mx > m[n] + kRaise ? mx : m[n];  // (each row by its own scores alone)
        const float f = __builtin_amdgcn_exp2f(m[n] - nm);
        m[n] = nm;
        l[n] *= f;
#pragma unroll
        for (int y = 0; y < NC; ++y) o[n][y] *= f;
#pragma unroll
        for (int y = 0; y < G; ++y) {
          if (!F32) ps[n][y] *= f;
          po[n][y] *= f;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[n][i] = __builtin_amdgcn_exp2f(fmaf(p[n][i], c, -m[n]));
        l[n] += p[n][i];
      }
    }

    const bf16x8 one = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f,
                        (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int y = 0; y < G; ++y) {
      const bf16x8 v0 = code_operand<F32>(x.v[2 * y]), v1 = code_operand<F32>(x.v[2 * y + 1]);
      f32x4 zs[2], zo[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        zs[u] = *reinterpret_cast<const f32x4*>(sc + 32 * G + 32 * y + 16 * u + 4 * m4);
        zo[u] = *reinterpret_cast<const f32x4*>(of + 32 * G + 32 * y + 16 * u + 4 * m4);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float f[8], sum = po[n][y];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[i] = p[n][i] * zs[i >> 2][i & 3];
          if (M) {
            // what a row does not see has weight 0, and may be NaN
            const bool seen = t0 + 16 * (i >> 2) + 4 * m4 + (i & 3) <= last[n];
            f[i] = seen ? f[i] : 0.0f;
            sum = seen ? fmaf(p[n][i], zo[i >> 2][i & 3], sum) : sum;
          } else {
            sum = fmaf(p[n][i], zo[i >> 2][i & 3], sum);
          }
        }
        po[n][y] = sum;
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
          if (!F32) ps[n][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, pw.v, ps[n][y], 0, 0, 0);
          o[n][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pw.v, o[n][2 * y], 0, 0, 0);
          o[n][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pw.v, o[n][2 * y + 1], 0, 0, 0);
        }
      }
    }
  };
  auto any_block = [&](const Block<D>& x, int t0) {
    const bool in = (unsigned)x.page < (unsigned)a.n_pages;
    if (!in || t0 + 31 > first_last || t0 + 32 > hi)
      block(Flag<true>(), x, t0, in);
    else
      block(Flag<false>(), x, t0, true);
  };
  for (; t0 < hi; t0 += 32 * NW) {
    load(x1, t0 + 32 * NW, next_page);
    next_page = page_of(t0 + 64 * NW);
    any_block(x0, t0);
    x0 = x1;
  }

  // the lane's rows: out of the codes' 16 (with the 8 of the moved offsets), the
  // offsets of all lanes' tokens
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] = add_xor32(add_xor16(l[n]));
#pragma unroll
    for (int y = 0; y < G; ++y) {
      const float x = add_xor32(add_xor16(po[n][y]));
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][2 * y + z][i] += F32 ? x : fmaf(-24.0f, ps[n][y][i], x);
    }
    if (m4 == 0) {
      sm[wave][16 * n + col] = m[n];
      sl[wave][16 * n + col] = l[n];
    }
  }
  __syncthreads();
  // join the waves: their sums against the common maximum to LDS, [wave][row][channel]
  // with 16-byte chunk x of row r at slot x ^ (r % 16), so that the 16 rows a write
  // touches lie on distinct banks; then four channels of a row a thread
  f32x4* sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 16 * n + col;
    float mm = sm[0][r];
#pragma unroll
    for (int x = 1; x < NW; ++x) mm = fmaxf(mm, sm[x][r]);
    const float f = __builtin_amdgcn_exp2f(m[n] - mm);
#pragma unroll
    for (int y = 0; y < NC; ++y) sums[(wave * R + r) * (D / 4) + ((4 * y + m4) ^ col)] = o[n][y] * f;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R * D / 4 / (64 * NW); ++i) {
    const int at = threadIdx.x + i * 64 * NW, rl = at / (D / 4), ch = at % (D / 4);
    const int r = row0 + rl;
    if (r >= n_rows) continue;
    float mm = sm[0][rl], lt = 0.0f;
    f32x4 v = {};
#pragma unroll
    for (int y = 1; y < NW; ++y) mm = fmaxf(mm, sm[y][rl]);
#pragma unroll
    for (int y = 0; y < NW; ++y) {
      v += sums[(y * R + rl) * (D / 4) + (ch ^ (rl & 15))];
      lt = fmaf(sl[y][rl], __builtin_amdgcn_exp2f(sm[y][rl] - mm), lt);
    }
    if (s.parts[b] == 1) {
      const int token = r / s.G, g = r - token * s.G;
      const long long to = s.o_off[b] + (long long)token * a.io.o_st +
                           (long long)(it.h * s.G + g) * a.io.o_sh + 4 * ch;
      v *= lt > 0.0f || lt != lt ? 1.0f / lt : 0.0f;
      if (F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.io.out) + to) = v;
      } else {
        const u32x2 x = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.io.out) + to) = x;
      }
      if (ch == 0 && a.io.lse)
        a.io.lse[(long long)(s.row0[b] + token) * (s.H * s.G) + it.h * s.G + g] =
            lt == 0.0f ? -INFINITY : (mm + log2f(lt)) * 0.6931471805599453f;
    } else {
      const long long slot = s.part0[b] + ((long long)it.h * n_rows + r) * s.parts[b] + it.part;
      *reinterpret_cast<f32x4*>(a.io.part + slot * D + 4 * ch) = v;
      if (ch == 0) {
        a.io.ml[2 * slot] = mm;
        a.io.ml[2 * slot + 1] = lt;
      }
    }
  }
}

template <int D>
hipError_t launch(int dtype, const AttnShape& sh, const PagedAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.s.item0[a.s.B] * a.s.H));
  const int threads = kPagedWaves * 64;
  if (dtype == HF_F32) {
    if (sh.rows == 16) paged_attention_kernel<D, 1, true><<<grid, threads, 0, st>>>(a);
    else paged_attention_kernel<D, 2, true><<<grid, threads, 0, st>>>(a);
  } else {
    if (sh.rows == 16) paged_attention_kernel<D, 1, false><<<grid, threads, 0, st>>>(a);
    else paged_attention_kernel<D, 2, false><<<grid, threads, 0, st>>>(a);
  }
  return hipGetLastError();
}

// Heads a workgroup: with many blocks to do all of them, so that the angles of a
// block are formed once.
int heads_per_workgroup(const PagedRowsArgs& a) {
  return (int64_t)a.blk0[a.B] * a.n_layers * a.H >= 4096 ? a.H : 1;
}

}  // namespace

AttnShape paged_shape(int dtype, int d_h, int64_t max_rows) {
  AttnShape sh;
  sh.rows = max_rows <= 16 ? 16 : 32;
  sh.by_keys = 1;
  sh.wg_target = 512;
  sh.step = 32 * kPagedWaves;
  sh.join_keys = 512;
  return sh;
}

hipError_t launch_paged_attention(int dtype, int d_h, const AttnShape& sh, const PagedAttnArgs& a,
                                  hipStream_t s) {
  return d_h == 128 ? launch<128>(dtype, sh, a, s) : launch<64>(dtype, sh, a, s);
}

hipError_t launch_paged_append(int dtype, int d_h, const PagedRowsArgs& a, hipStream_t s) {
  const int hpw = heads_per_workgroup(a);
  const dim3 grid((unsigned)(a.blk0[a.B] * ((a.H + hpw - 1) / hpw)), 2, (unsigned)a.n_layers);
  if (dtype == HF_BF16) {
    if (d_h == 128) paged_append_kernel<uint16_t, 128><<<grid, 256, 0, s>>>(a, hpw);
    else paged_append_kernel<uint16_t, 64><<<grid, 128, 0, s>>>(a, hpw);
  } else {
    if (d_h == 128) paged_append_kernel<float, 128><<<grid, 256, 0, s>>>(a, hpw);
    else paged_append_kernel<float, 64><<<grid, 128, 0, s>>>(a, hpw);
  }
  return hipGetLastError();
}

hipError_t launch_paged_read(int dtype, int d_h, const PagedRowsArgs& a, hipStream_t s) {
  const int hpw = heads_per_workgroup(a);
  const dim3 grid((unsigned)(a.blk0[a.B] * ((a.H + hpw - 1) / hpw)), 2, (unsigned)a.n_layers);
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
