// The attention weight that each key gets from a run of queries, from the log-sum-exps of
// their attention:
//
//   w_j = decay prior_j + sum over heads g of the group and rows i that see j of
//         exp(scale <q_ig, k_j> - lse_ig)
//
// over dense keys and over the paged cache held in 4 bits.  The keys stand still: a wave
// holds a tile of them in registers as one operand of its matrix instructions and takes the
// query rows past them, tile after tile.  With S = Q K^T a lane has scores of one key, so
// that a key's sum over the rows is a sum over the lane's registers, one number a key and
// lane, joined at the end.  No score leaves the registers, nothing is joined by atomics, and
// the order of the sums depends on the lengths alone.
//
// A row's lse is wanted in the registers of its scores, rows down the registers: a matrix
// instruction with ones spreads it there, as three bf16 terms of 8 bits each (as it is in
// fp32), exactly.
#include <hip/hip_runtime.h>

#include "hf_paged.h"

namespace hf {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// Rows whose lse lies past this are taken with the masked ones, where an exponent above 0,
// which only the rounding of the lse can make, counts as 0.  (Below it that rounding is under
// 2^-11: a weight passes 1 by as much at most.)
constexpr float kFarLse = 4096.0f;

// x, spread over A's row of the lane's column: what an instruction with ones() makes of it.
FI bf16x8 spread(float x, bool mine) {
  float p[3];
  split<3>(x, p);
  if (!finite_bits(x)) p[1] = p[2] = 0.0f;
  bf16x8 a = {};
  if (mine) {
    a[0] = (__bf16)p[0];
    a[1] = (__bf16)p[1];
    a[2] = (__bf16)p[2];
  }
  return a;
}
FI bf16x8 ones(bool mine) {
  bf16x8 a = {};
  if (mine) a[0] = a[1] = a[2] = (__bf16)1.0f;
  return a;
}

// 32 rows (queries or keys) as an operand of 32 x 32 products, a lane the row lane % 32.
template <int D_>
struct RowsBf16 {
  static constexpr int D = D_;
  typedef uint16_t T;
  bf16x8 f[D / 16];
  FI void load(const T* row, int lane) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) f[c] = *reinterpret_cast<const bf16x8*>(row + 16 * c + 8 * (lane >> 5));
  }
  FI static f32x16 product(const RowsBf16& q, const RowsBf16& k) {
    f32x16 s = {};
#pragma unroll
    for (int c = 0; c < D / 16; ++c) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q.f[c], k.f[c], s, 0, 0, 0);
    return s;
  }
  FI static f32x16 by_rows(float x, int lane) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(spread(x, lane < 32), ones(lane < 32), f32x16{}, 0, 0, 0);
  }
};
// Step (u, j) takes channels 8 u + j and 8 u + 4 + j, so that a lane loads 16 bytes.
template <int D_>
struct RowsF32 {
  static constexpr int D = D_;
  typedef float T;
  f32x4 f[D / 8];
  FI void load(const T* row, int lane) {
#pragma unroll
    for (int u = 0; u < D / 8; ++u) f[u] = *reinterpret_cast<const f32x4*>(row + 8 * u + 4 * (lane >> 5));
  }
  FI static f32x16 product(const RowsF32& q, const RowsF32& k) {
    f32x16 s = {};
#pragma unroll
    for (int u = 0; u < D / 8; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q.f[u][j], k.f[u][j], s, 0, 0, 0);
    return s;
  }
  FI static f32x16 by_rows(float x, int lane) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(lane < 32 ? x : 0.0f, 1.0f, f32x16{}, 0, 0, 0);
  }
};

struct WeighItem {
  int b, h, i;       // i: the item's number in its sequence and head
  int n, t, rows, row0, key0;
};
FI WeighItem weigh_item(const WeighArgs& a) {
  WeighItem it;
  int i = divide(blockIdx.x, a.by_h);
  it.h = blockIdx.x - i * a.H;
  it.b = find_seq(a.s, &WeighSeq::item0, a.B, i);
  const WeighSeq s = a.s[it.b];
  it.i = i - s.item0;
  it.n = s.n;
  it.t = s.t;
  it.rows = s.n * a.G;
  it.row0 = s.row0;
  it.key0 = s.key0;
  return it;
}
// The first row that sees a key (rows of a head: token * G + head of the group).
FI int first_row(const WeighArgs& a, const WeighItem& it, int key) {
  return a.causal ? max(key - (it.t - it.n), 0) * a.G : 0;
}
FI long long query_at(const WeighArgs& a, const WeighItem& it, int r, float& lse) {
  const int token = divide(r, a.by_g), head = it.h * a.G + r - token * a.G;
  lse = a.lse[(long long)(it.row0 + token) * (a.H * a.G) + head];
  return seq_at(it.b, it.row0, a.q_sb, a.q_st) + token * a.q_st + head * a.q_sh;
}
FI void write_weight(const WeighArgs& a, const WeighItem& it, int key, float w) {
  if (a.prior) w = fmaf(a.decay, a.prior[it.b * a.p_sb + it.h * a.p_sh + key], w);
  a.out[it.b * a.o_sb + it.h * a.o_sh + key] = w;
}

// The sum of N weights, by halves.
template <int N>
FI float sum_of(float (&x)[N]) {
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] += x[i + n];
  return x[0];
}

// KB blocks of 32 keys a wave; KW waves with keys of their own, RW waves that share the rows.
template <class R, int KB, int KW, int RW>
__global__ __launch_bounds__(64 * KW * RW, 2) void attention_weights_kernel(const WeighArgs a) {
  typedef typename R::T T;
  constexpr int KT = 32 * KB;
  __shared__ float sums[RW > 1 ? RW : 1][KW * KT];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave / RW, rw = wave % RW;
  const WeighItem it = weigh_item(a);
  const int t0 = (it.i * KW + kw) * KT;
  float acc[KB] = {};
  if (t0 < it.t) {  // (a wave without keys waits at the end)
    const T* kb = static_cast<const T*>(a.k) + seq_at(it.b, it.key0, a.k_sb, a.k_st) + it.h * a.k_sh;
    R k[KB];
    int see[KB];  // the first row that sees the lane's key
#pragma unroll
    for (int y = 0; y < KB; ++y) {
      const int key = min(t0 + 32 * y + (lane & 31), it.t - 1);
      k[y].load(kb + key * a.k_st, lane);
      see[y] = first_row(a, it, key);
    }
    const int all = first_row(a, it, min(t0 + KT, it.t) - 1);  // from here on rows see all of the keys
    const T* q0 = static_cast<const T*>(a.q);
    const int first = first_row(a, it, t0) / 32 * 32 + 32 * rw;
    R q;
    float lse = 0.0f;
    auto fetch = [&](int r0) {
      if (r0 >= it.rows) return;
      const long long at = query_at(a, it, min(r0 + (lane & 31), it.rows - 1), lse);
      q.load(q0 + at, lane);
    };
    fetch(first);
    for (int r0 = first; r0 < it.rows; r0 += 32 * RW) {
      const float x = -lse * kLog2e;
      const f32x16 nl = R::by_rows(x, lane);
      const bool far = __any(!(fabsf(x) <= kFarLse));
      f32x16 s[KB];
#pragma unroll
      for (int y = 0; y < KB; ++y) s[y] = R::product(q, k[y]);
      fetch(r0 + 32 * RW);
      if (!far && r0 >= all && r0 + 32 <= it.rows) {
#pragma unroll
        for (int y = 0; y < KB; ++y) {
          float w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(s[y][i], a.c, nl[i]));
          acc[y] += sum_of(w);
        }
      } else {
#pragma unroll
        for (int y = 0; y < KB; ++y) {
          float w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = r0 + 8 * (i >> 2) + 4 * half + (i & 3);
            const float e = fmaf(s[y][i], a.c, nl[i]);
            w[i] = r >= see[y] && r < it.rows ? __builtin_amdgcn_exp2f(e > 0.0f ? 0.0f : e) : 0.0f;
          }
          acc[y] += sum_of(w);
        }
      }
    }
  }
#pragma unroll
  for (int y = 0; y < KB; ++y) acc[y] = add_xor32(acc[y]);
  if (RW == 1) {
#pragma unroll
    for (int y = 0; y < KB; ++y) {
      const int key = t0 + 32 * y + lane;
      if (lane < 32 && key < it.t) write_weight(a, it, key, acc[y]);
    }
    return;
  }
#pragma unroll
  for (int y = 0; y < KB; ++y)
    if (lane < 32) sums[rw][kw * KT + 32 * y + lane] = acc[y];
  __syncthreads();
  for (int x = threadIdx.x; x < KW * KT; x += 64 * KW * RW) {
    const int key = it.i * KW * KT + x;
    float w = 0.0f;
#pragma unroll
    for (int y = 0; y < RW; ++y) w += sums[y][x];
    if (key < it.t) write_weight(a, it, key, w);
  }
}

// Over the pages: 16 NU tokens a wave, on v_mfma_f32_16x16x32_bf16 with the codes as they are
// stored (the arithmetic of scales and offsets is that of the attention over the pages), 16
// query rows at a time.  The lane has tokens lane % 16 of each 16 and, with m = lane / 16,
// rows 4 m + i.
template <int D, bool F32, int NU>
__global__ __launch_bounds__(256, 2) void paged_weights_kernel(const WeighArgs a) {
  constexpr int G = D / 32, S = F32 ? 3 : 1, KT = 16 * NU;
  const int lane = threadIdx.x & 63, col = lane & 15, m4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WeighItem it = weigh_item(a);
  const int t0 = (it.i * 4 + wave) * KT;
  if (t0 >= it.t) return;
  const PageHead<D> ph(a.log2_page);
  const int32_t* table = a.table + it.b * a.table_stride;
  // the codes and words of all tokens on their way at once
  uint32_t code[NU][G], word[NU][G];
  bool in[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int tok = t0 + 16 * u;
    const int page = tok < it.t ? table[tok >> a.log2_page] : -1;
    in[u] = (unsigned)page < (unsigned)a.n_pages;  // (a hole loads from page 0 and counts as 0)
    const uint8_t* head = a.pages + (long long)(in[u] ? page : 0) * a.page_bytes + (long long)it.h * ph.bytes();
    const int row = (in[u] ? tok & (ph.P - 1) : 0) + col;
    const uint8_t* c = head + ph.kcode(row) + m4 * (4 * G);
    const uint8_t* w = head + ph.word(0, row);
    if (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(c), y = *reinterpret_cast<const u32x4*>(w);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        code[u][g] = x[g & 3];
        word[u][g] = y[g & 3];
      }
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(c), y = *reinterpret_cast<const u32x2*>(w);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        code[u][g] = x[g & 1];
        word[u][g] = y[g & 1];
      }
    }
  }
  int see[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) see[u] = first_row(a, it, min(t0 + 16 * u + col, it.t - 1));
  const int all = first_row(a, it, min(t0 + KT, it.t) - 1);
  const int first = first_row(a, it, t0) / 16 * 16;

  typedef uint32_t QRaw[F32 ? 8 : 4];
  QRaw raw[G];
  float lse = 0.0f;
  auto fetch = [&](int r0) {
    if (r0 >= it.rows) return;
    const long long at = query_at(a, it, min(r0 + col, it.rows - 1), lse);
    const uint8_t* row = static_cast<const uint8_t*>(a.q) + at * (F32 ? 4 : 2);
#pragma unroll
    for (int y = 0; y < G; ++y) load_dwords<F32 ? 8 : 4>(row + (32 * y + 8 * m4) * (F32 ? 4 : 2), raw[y]);
  };
  fetch(first);
  const Codes codes;
  bf16x8 kc[NU][G];
  float acc[NU] = {};
#pragma unroll
  for (int u = 0; u < NU; ++u)
#pragma unroll
    for (int g = 0; g < G; ++g) kc[u][g] = codes.operand<F32>(code[u][g]);
  for (int r0 = first; r0 < it.rows; r0 += 16) {
    bf16x8 q[S][G];
    bf16x8 qo = {};  // against the words: the sums of the groups, in three terms
#pragma unroll
    for (int y = 0; y < G; ++y) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = raw[y][F32 ? e : e / 2];
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
    const float x = -lse * kLog2e;
    const f32x4 nl =
        __builtin_amdgcn_mfma_f32_16x16x32_bf16(spread(x, lane < 16), ones(lane < 16), f32x4{}, 0, 0, 0);
    const bool plain = !__any(!(fabsf(x) <= kFarLse)) && r0 >= all && r0 + 16 <= it.rows;
    fetch(r0 + 16);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      union {
        uint32_t d[4];
        bf16x8 v;
      } wk = {{0, 0, 0, 0}};
#pragma unroll
      for (int y = 0; y < G; ++y) wk.d[y] = word[u][y];
      f32x4 v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qo, wk.v, f32x4{}, 0, 0, 0);
#pragma unroll
      for (int y = 0; y < G; ++y) {
        f32x4 d = {};
#pragma unroll
        for (int z = 0; z < S; ++z) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[z][y], kc[u][y], d, 0, 0, 0);
        const float ks = __builtin_bit_cast(float, word[u][y] & 0xffff0000u);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(ks, d[i], v[i]);
      }
      float w[4];
      if (plain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(v[i], a.c, nl[i]));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = r0 + 4 * m4 + i;
          const float e = fmaf(v[i], a.c, nl[i]);
          w[i] = r >= see[u] && r < it.rows ? __builtin_amdgcn_exp2f(e > 0.0f ? 0.0f : e) : 0.0f;
        }
      }
      acc[u] += sum_of(w);
    }
  }
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const float w = add_xor32(add_xor16(acc[u]));
    const int key = t0 + 16 * u + col;
    if (m4 == 0 && key < it.t) write_weight(a, it, key, in[u] ? w : 0.0f);
  }
}

constexpr int kPagedTokens = 64;  // a wave

template <class R, int KB, int KW, int RW>
void launch_as(const WeighArgs& a, hipStream_t s) {
  attention_weights_kernel<R, KB, KW, RW><<<(unsigned)(a.n_items * a.H), 64 * KW * RW, 0, s>>>(a);
}

template <int D>
void launch(int dtype, const WeighShape& sh, const WeighArgs& a, hipStream_t s) {
  if (dtype == HF_F32) {
    if (sh.row_waves > 1) launch_as<RowsF32<D>, 1, 1, 8>(a, s);
    else launch_as<RowsF32<D>, 1, 4, 1>(a, s);
  } else if (sh.row_waves > 1) {
    if (sh.keys == 128) launch_as<RowsBf16<D>, 4, 1, 8>(a, s);
    else launch_as<RowsBf16<D>, 2, 1, 8>(a, s);
  } else {
    launch_as<RowsBf16<D>, 2, 4, 1>(a, s);
  }
}

}  // namespace

// Keys of a work item and the waves that share its rows.
WeighShape weigh_shape(int dtype, bool paged, int64_t heads, int64_t keys, int64_t rows) {
  WeighShape sh;
  if (paged) {
    sh.row_waves = 1;
    sh.keys = 4 * kPagedTokens;
    return sh;
  }
  const int wave = dtype == HF_F32 ? 32 : 64;
  sh.row_waves = rows >= 8 * 32 ? 8 : 1;
  sh.keys = sh.row_waves == 1 ? 4 * wave : wave;
  if (dtype == HF_BF16 && sh.row_waves == 8 && keys / 128 * heads >= 256) sh.keys = 128;
  return sh;
}

hipError_t launch_attention_weights(int dtype, int d_h, const WeighShape& sh, const WeighArgs& a, hipStream_t s) {
  if (d_h == 128)
    launch<128>(dtype, sh, a, s);
  else
    launch<64>(dtype, sh, a, s);
  return hipGetLastError();
}

hipError_t launch_paged_weights(int dtype, int d_h, const WeighArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n_items * a.H);
  constexpr int NU = kPagedTokens / 16;
  if (d_h == 128) {
    if (dtype == HF_F32) paged_weights_kernel<128, true, NU><<<grid, 256, 0, s>>>(a);
    else paged_weights_kernel<128, false, NU><<<grid, 256, 0, s>>>(a);
  } else {
    if (dtype == HF_F32) paged_weights_kernel<64, true, NU><<<grid, 256, 0, s>>>(a);
    else paged_weights_kernel<64, false, NU><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace hf
