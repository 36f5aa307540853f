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

#include <algorithm>
#include <cmath>

#include "hf_paged.h"

namespace hf {
namespace {

// (lambdas whose arguments have to stay in registers)
#define INLINE __attribute__((always_inline))

constexpr float kLog2e = 1.44269504088896340736f;

// Rows whose lse lies past this are taken with the masked ones, where an exponent above 0,
// which only the rounding of the lse can make, counts as 0.  (Below it that rounding is under
// 2^-11: a weight passes 1 by as much at most.)
constexpr float kFarLse = 4096.0f;

// x as the three bf16 terms that make it, packed; what is not finite as one.
FI u32x2 terms(float x) {
  float p[3];
  split<3>(x, p);
  if (!finite_bits(x)) p[1] = p[2] = 0.0f;
  return u32x2{pack_bf16(p[0], p[1]), pack_bf16(p[2], 0.0f)};
}
// Operands whose product has the first one's terms, of row lane % 32 (16), in every column.
FI bf16x8 spread(u32x2 t, bool mine) {
  union {
    uint32_t u[4];
    bf16x8 v;
  } a = {{mine ? t[0] : 0u, mine ? t[1] : 0u, 0u, 0u}};
  return a.v;
}
FI bf16x8 ones(bool mine) {
  bf16x8 a = {};
  if (mine) a[0] = a[1] = a[2] = (__bf16)1.0f;
  return a;
}

// 32 rows (queries or keys) as an operand of 32 x 32 products, a lane the row lane % 32, in
// steps of 16 bytes a lane.
template <int D_>
struct RowsBf16 {
  static constexpr int D = D_, STEPS = D / 16, MFMAS = 1;  // products a step
  static constexpr int WAVES = 2, CHAINS = 2;               // a SIMD; sums that a wave forms at once
  static constexpr int ROWB = 2 * D;                        // bytes of a row
  typedef uint16_t T;
  typedef bf16x8 F;
  typedef u32x2 L;  // a row's -lse as by_rows takes it
  F f[STEPS];
  // Where 16-byte chunk c of row r lies in a row of LDS: 32 rows are read at once.
  FI static int slot(int r, int c) { return c ^ (D == 128 ? r & 15 : (r >> 1) & 7); }
  FI static F read(const unsigned char* st, int lane, int c) {
    const int r = lane & 31;
    return *reinterpret_cast<const F*>(st + r * ROWB + slot(r, 2 * c + (lane >> 5)) * 16);
  }
  FI void load(const T* row, int lane) {
#pragma unroll
    for (int c = 0; c < STEPS; ++c) f[c] = *reinterpret_cast<const F*>(row + 16 * c + 8 * (lane >> 5));
  }
  FI static f32x16 step(F q, F k, f32x16 s) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k, s, 0, 0, 0); }
  FI static L hold(float x) { return terms(x); }
  FI static f32x16 by_rows(L x, int lane) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(spread(x, lane < 32), ones(lane < 32), f32x16{}, 0, 0, 0);
  }
};
// Step u, product j takes channels 8 u + j and 8 u + 4 + j.
template <int D_>
struct RowsF32 {
  static constexpr int D = D_, STEPS = D / 8, MFMAS = 4;
  static constexpr int WAVES = 2, CHAINS = 2;
  static constexpr int ROWB = 4 * D;
  typedef float T;
  typedef f32x4 F;
  typedef float L;
  F f[STEPS];
  FI static int slot(int r, int c) { return c ^ (r & 15); }
  FI static F read(const unsigned char* st, int lane, int u) {
    const int r = lane & 31;
    return *reinterpret_cast<const F*>(st + r * ROWB + slot(r, 2 * u + (lane >> 5)) * 16);
  }
  FI void load(const T* row, int lane) {
#pragma unroll
    for (int u = 0; u < STEPS; ++u) f[u] = *reinterpret_cast<const F*>(row + 8 * u + 4 * (lane >> 5));
  }
  FI static f32x16 step(F q, F k, f32x16 s) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q[j], k[j], s, 0, 0, 0);
    return s;
  }
  FI static L hold(float x) { return x; }
  FI static f32x16 by_rows(L x, int lane) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(lane < 32 ? x : 0.0f, 1.0f, f32x16{}, 0, 0, 0);
  }
};

struct WeighItem {
  int b, h, i;       // i: the tile's number in its sequence
  int n, t, rows, row0, key0;
  int part;          // of the rows
};
// Work items are tiles (the join's, and all where the rows are not cut), or the pairs of a part
// of the rows and a tile that some of them see: the last part's first, which sees the most.
FI WeighItem weigh_item(const WeighArgs& a, bool tiles) {
  WeighItem it;
  int i = divide(blockIdx.x, a.by_h);
  it.h = blockIdx.x - i * a.H;
  it.b = tiles ? find_seq(a.s, &WeighSeq::tile0, a.B, i) : find_seq(a.s, &WeighSeq::item0, a.B, i);
  const WeighSeq s = a.s[it.b];
  it.n = s.n;
  it.t = s.t;
  it.rows = s.n * a.G;
  it.row0 = s.row0;
  it.key0 = s.key0;
  it.part = 0;
  it.i = i - (tiles ? s.tile0 : s.item0);
  if (!tiles && s.parts > 1) {
    const int lane = threadIdx.x & 63;
    for (int x = 0;; x += 64) {
      const int p = s.parts - 1 - x - lane;
      const int mine = p < 0 ? 0 : weigh_tiles(s, a.G, a.chunk, a.tile, a.causal, p);
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      const unsigned long long past = __ballot(upto > it.i);
      if (past) {
        const int l = __builtin_ctzll(past);
        it.part = s.parts - 1 - x - l;
        it.i -= __builtin_amdgcn_readlane(upto - mine, l);
        break;
      }
      it.i -= __builtin_amdgcn_readlane(upto, 63);
    }
  }
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

template <bool M>
struct Flag {
  static constexpr bool value = M;
};

// Many rows: NW waves with KB blocks of 32 keys each, all against the same rows, which come
// through two LDS stages of 64 rows, on their way in registers two stages ahead.  Where there are
// too few tiles of keys to fill the chip the rows of each are cut into parts as well, whose sums
// weights_join_kernel adds; of a causal mask only the pairs of a part and a tile are workgroups
// in which some row sees some key (one that ends at once still keeps its CU for a while).
// The products and the exponentials, 16 cycles a wave each, bound it: a prompt of 8,192 tokens,
// 32 / 8 heads of 128, takes 327 to 383 us by card, 0.73 to 0.85 PFLOP/s, where the products alone
// would take some 200, and one of 2,048 42 us (with the rows in one piece 155).
// Two waves a SIMD fill part of each other's phases.  Taking both in turn within a wave would
// do better (in a loop of nothing else 1,450 cycles for what takes 2,205 in two waves), but with
// a second block's scores and operands the keys no longer fit in registers: 450 us and more.
// Each wave with rows of its own loads (no LDS) took 450 us.
// fp32: 2,001 tokens, 14 / 2 heads of 64, 53 us, at half the rate of the fp32 products; 161 before
// the rows went through LDS in parts.
template <class R, int KB, int NW>
__global__ __launch_bounds__(64 * NW, R::WAVES) void weights_rows_kernel(const WeighArgs a) {
  typedef typename R::T T;
  constexpr int KT = 32 * KB, RS = 64, CPR = R::ROWB / 16, NB = RS * CPR / 64 / NW;
  static_assert(NB * 64 * NW == RS * CPR, "whole loads a wave");
  struct Stage {
    __attribute__((aligned(1024))) unsigned char q[RS * R::ROWB];
    typename R::L lse[RS];
    int far;
  };
  __shared__ Stage st0, st1;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WeighItem it = weigh_item(a, false);
  const int tile0 = it.i * NW * KT, t0 = tile0 + wave * KT;
  // the part's rows: whole stages
  const int row0 = max(first_row(a, it, tile0) / RS * RS, it.part * a.chunk);
  const int end = min(it.rows, (int)min((long long)it.rows, (it.part + 1ll) * a.chunk));

  // A lane's rows of the next stage: the row's number in the stage stays, its token and head
  // move on by a stage's rows.  (Row r is token r / G and head r % G of the group.)
  struct Place {
    int g;
    long long at;  // elements to the row, of q or lse
  };
  const T* q = static_cast<const T*>(a.q) + seq_at(it.b, it.row0, a.q_sb, a.q_st) + it.h * a.G * a.q_sh;
  const float* lse = a.lse + (long long)it.row0 * (a.H * a.G) + it.h * a.G;
  const long long lse_st = a.H * a.G;
  const int step_t = divide(RS, a.by_g), step_g = RS - step_t * a.G;
  Place qp[NB], lp;
  auto place = [&](Place& p, int r, long long st, long long sh) INLINE {
    const int token = divide(r, a.by_g);
    p.g = r - token * a.G;
    p.at = token * st + p.g * sh;
  };
  auto advance = [&](Place& p, long long st, long long sh) INLINE {
    p.g += step_g;
    p.at += step_t * st + step_g * sh;
    if (p.g >= a.G) {
      p.g -= a.G;
      p.at += st - a.G * sh;
    }
  };
  const int my_row = wave * NB * (64 / CPR) + lane / CPR;  // of a stage; the next ones 64 / CPR further
#pragma unroll
  for (int i = 0; i < NB; ++i) place(qp[i], row0 + my_row + i * (64 / CPR), a.q_st, a.q_sh);
  place(lp, row0 + lane, lse_st, 1);
  // The rows from r0 on on their way (of rows behind the last one: the first one, which is
  // there), and to LDS.
  struct Raw {
    u32x4 q[NB];
    float lse;
  };
  auto load = [&](int r0, Raw& raw) INLINE {
    if (r0 >= end) return;
    if (r0 + RS > it.rows) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (r0 + my_row + i * (64 / CPR) >= it.rows) qp[i].at = 0;
      if (r0 + lane >= it.rows) lp.at = 0;
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      raw.q[i] = *reinterpret_cast<const u32x4*>(q + qp[i].at + lane % CPR * (16 / (int)sizeof(T)));
      advance(qp[i], a.q_st, a.q_sh);
    }
    if (wave == 0) {
      raw.lse = lse[lp.at];
      advance(lp, lse_st, 1);
    }
  };
  auto put = [&](Stage& st, const Raw& raw) INLINE {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int r = my_row + i * (64 / CPR);
      *reinterpret_cast<u32x4*>(st.q + r * R::ROWB + R::slot(r, lane % CPR) * 16) = raw.q[i];
    }
    if (wave == 0) {
      const float x = -raw.lse * kLog2e;
      st.lse[lane] = R::hold(x);
      const bool far = __any(!(fabsf(x) <= kFarLse));
      if (lane == 0) st.far = far;
    }
  };
  auto meet = [&]() INLINE {  // what the waves wrote is there, and none reads what is written next
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  float acc[KB] = {};
  if (row0 < end) {
    Raw ra, rb;
    load(row0, ra);
    const T* kb = static_cast<const T*>(a.k) + seq_at(it.b, it.key0, a.k_sb, a.k_st) + it.h * a.k_sh;
    R k[KB];
    int see[KB];  // the first row that sees the lane's key
#pragma unroll
    for (int y = 0; y < KB; ++y) {
      const int key = min(t0 + 32 * y + (lane & 31), it.t - 1);
      k[y].load(kb + key * a.k_st, lane);
      see[y] = first_row(a, it, key);
    }
    // (waited for here: a wait for the keys in the loop waits for the rows in flight as well)
#pragma unroll
    for (int y = 0; y < KB; ++y)
#pragma unroll
      for (int c = 0; c < R::STEPS; ++c) asm volatile("" : "+v"(k[y].f[c]));
    const int all = first_row(a, it, min(t0 + KT, it.t) - 1);  // from here on rows see all of the keys
    const int some = first_row(a, it, min(t0, it.t - 1));      // from here on rows see some of them
    // 32 rows from r0 on, the stage's i-th.  edge: some row may not see some key; care: it may
    // lie behind the last one, or far away.
    auto turn = [&](auto edge, auto care, int r0, const Stage& st, int i) INLINE {
      const f32x16 nl = R::by_rows(st.lse[32 * i + (lane & 31)], lane);
      // A matrix instruction waits for the one before it that adds to the same numbers for longer
      // than it takes: CH sums a block, of every CH-th step.
      constexpr int CH = R::CHAINS / KB;
      f32x16 s[KB], sum[CH][KB] = {};
#pragma unroll
      for (int c = 0; c < R::STEPS; ++c) {
        const typename R::F f = R::read(st.q + i * 32 * R::ROWB, lane, c);
#pragma unroll
        for (int y = 0; y < KB; ++y) sum[c % CH][y] = R::step(f, k[y].f[c], sum[c % CH][y]);
      }
#pragma unroll
      for (int y = 0; y < KB; ++y) {
        s[y] = sum[0][y];
#pragma unroll
        for (int x = 1; x < CH; ++x) s[y] += sum[x][y];
      }
#pragma unroll
      for (int y = 0; y < KB; ++y) {
        float w[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = r0 + 8 * (j >> 2) + 4 * half + (j & 3);
          float e = fmaf(s[y][j], a.c, nl[j]);
          if (decltype(care)::value) e = e > 0.0f ? 0.0f : e;
          if (decltype(edge)::value) e = r >= see[y] ? e : -INFINITY;
          if (decltype(care)::value) e = r < end ? e : -INFINITY;
          w[j] = __builtin_amdgcn_exp2f(e);
        }
        acc[y] += sum_of(w);
      }
    };
    // (raw: the rows of the next stage)
    auto stage = [&](int r0, Stage& st, Stage& next, Raw& raw) INLINE {
      meet();
      if (r0 + RS < end) put(next, raw);
      load(r0 + 3 * RS, raw);
      if (t0 >= it.t) return;
      const bool care = st.far || r0 + RS > end;
#pragma unroll 1
      for (int i = 0, r = r0; i < 2; ++i, r += 32) {
        if (r + 32 <= some) continue;
        if (care) turn(Flag<true>(), Flag<true>(), r, st, i);
        else if (r < all) turn(Flag<true>(), Flag<false>(), r, st, i);
        else turn(Flag<false>(), Flag<false>(), r, st, i);
      }
    };
    put(st0, ra);
    load(row0 + RS, ra);
    load(row0 + 2 * RS, rb);
    for (int r0 = row0; r0 < end; r0 += 2 * RS) {
      stage(r0, st0, st1, ra);
      if (r0 + RS < end) stage(r0 + RS, st1, st0, rb);
    }
  }
#pragma unroll
  for (int y = 0; y < KB; ++y) {
    const float w = add_xor32(acc[y]);
    const int key = t0 + 32 * y + lane;
    if (lane < 32 && key < it.t) {
      if (a.part) a.part[((long long)it.part * a.H + it.h) * a.keys + it.key0 + key] = w;
      else write_weight(a, it, key, w);
    }
  }
}

// The sums of the parts of each key's rows, in their order.
__global__ __launch_bounds__(256) void weights_join_kernel(const WeighArgs a) {
  const WeighItem it = weigh_item(a, true);
  const int parts = a.s[it.b].parts, first = first_row(a, it, it.i * a.tile) / a.chunk;
  for (int key = it.i * a.tile + threadIdx.x; key < min(it.t, (it.i + 1) * a.tile); key += 256) {
    float w = 0.0f;
#pragma unroll 4
    for (int p = first; p < parts; ++p) w += a.part[((long long)p * a.H + it.h) * a.keys + it.key0 + key];
    write_weight(a, it, key, w);
  }
}

// Few rows: four waves, each with KB blocks of 32 keys and all rows, which it loads for itself, the
// next 32 on their way.  Reading the keys bounds it: 16 single queries over 4,096 keys of 32 / 8
// heads of 128 each, 134 MB, 28 us, 4.8 TB/s.
template <class R, int KB>
__global__ __launch_bounds__(256, 2) void weights_few_kernel(const WeighArgs a) {
  typedef typename R::T T;
  constexpr int KT = 32 * KB;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WeighItem it = weigh_item(a, true);
  const int t0 = (it.i * 4 + wave) * KT;
  if (t0 >= it.t) return;
  const T* q0 = static_cast<const T*>(a.q);
  R q, k[KB];
  float lse = 0.0f;
  auto fetch = [&](int r0) {
    if (r0 >= it.rows) return;
    const long long at = query_at(a, it, min(r0 + (lane & 31), it.rows - 1), lse);
    q.load(q0 + at, lane);
  };
  const int first = first_row(a, it, t0) / 32 * 32;
  fetch(first);
  const T* kb = static_cast<const T*>(a.k) + seq_at(it.b, it.key0, a.k_sb, a.k_st) + it.h * a.k_sh;
  int see[KB];
#pragma unroll
  for (int y = 0; y < KB; ++y) {
    const int key = min(t0 + 32 * y + (lane & 31), it.t - 1);
    k[y].load(kb + key * a.k_st, lane);
    see[y] = first_row(a, it, key);
  }
  float acc[KB] = {};
  for (int r0 = first; r0 < it.rows; r0 += 32) {
    const f32x16 nl = R::by_rows(R::hold(-lse * kLog2e), lane);
    f32x16 s[KB] = {};
#pragma unroll
    for (int c = 0; c < R::STEPS; ++c)
#pragma unroll
      for (int y = 0; y < KB; ++y) s[y] = R::step(q.f[c], k[y].f[c], s[y]);
    fetch(r0 + 32);
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
#pragma unroll
  for (int y = 0; y < KB; ++y) {
    const float w = add_xor32(acc[y]);
    const int key = t0 + 32 * y + lane;
    if (lane < 32 && key < it.t) write_weight(a, it, key, w);
  }
}

// Over the pages: four waves of 16 NU tokens each, tile after tile, on v_mfma_f32_16x16x32_bf16
// with the codes as they are stored (the arithmetic of scales and offsets is that of the
// attention over the pages).  The lane has tokens lane % 16 of each 16 and, with m = lane / 16,
// rows 4 m + i of 16 query rows.  The query rows, 64 at a time, are brought into the form that
// the products take once for all tiles (each wave 16 of them) and lie in LDS; the codes of the
// next tile are on their way while one is worked on.  Four bits a value are little to read: what
// bounds long runs of queries are the products and exponentials (2,048 over 8,192 keys of 32 / 8
// heads 399 us; with the rows prepared by each wave for itself 582), what bounds single tokens
// is the way to the first codes (B = 16, up to 8,192 keys, 36 MB: 19.7 us; the loads alone 15).
// With 64 tokens a wave there are registers for half as many waves: 25.3 us.
template <int D, bool F32, int NU>
__global__ __launch_bounds__(256, F32 ? 2 : 4) void paged_weights_kernel(const WeighArgs a) {
  constexpr int G = D / 32, S = F32 ? 3 : 1, KT = 16 * NU, NQ = S * G + 2;
  __shared__ u32x4 rows[4][NQ][64];  // a block's operands, those of the words, minus lse
  __shared__ int far[4];
  const int lane = threadIdx.x & 63, col = lane & 15, m4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WeighItem it = weigh_item(a, true);
  const int begin = it.i * a.tile, end = min(it.t, begin + a.tile);
  const PageHead<D> ph(a.log2_page);
  const int32_t* table = a.table + it.b * a.table_stride;

  uint32_t code[NU][G], word[NU][G];
  bool in[NU];
  auto load = [&](int t0) INLINE {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int tok = t0 + 16 * u;
      const int page = tok < end ? table[tok >> a.log2_page] : -1;
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
  };
  // rows r0 .. r0 + 15 into the wave's block
  auto prepare = [&](int r0) INLINE {
    if (r0 >= it.rows) return;
    typedef uint32_t QRaw[F32 ? 8 : 4];
    QRaw raw[G];
    float lse;
    const long long at = query_at(a, it, min(r0 + col, it.rows - 1), lse);
    const uint8_t* row = static_cast<const uint8_t*>(a.q) + at * (F32 ? 4 : 2);
#pragma unroll
    for (int y = 0; y < G; ++y) load_dwords<F32 ? 8 : 4>(row + (32 * y + 8 * m4) * (F32 ? 4 : 2), raw[y]);
    bf16x8 qo = {};  // against the words: the sums of the groups, in three terms
#pragma unroll
    for (int y = 0; y < G; ++y) {
      bf16x8 q[S];
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = raw[y][F32 ? e : e / 2];
        const float f = __builtin_bit_cast(float, F32 ? w : e & 1 ? w & 0xffff0000u : w << 16);
        sum += f;
        float p[S];
        split<S>(f, p);
#pragma unroll
        for (int z = 0; z < S; ++z) q[z][e < 4 ? 2 * e : 2 * (e - 4) + 1] = (__bf16)p[z];
      }
#pragma unroll
      for (int z = 0; z < S; ++z) rows[wave][z * G + y][lane] = __builtin_bit_cast(u32x4, q[z]);
      sum = add_xor32(add_xor16(sum));
      float p[3];
      split<3>(sum, p);
      const float mine = m4 == 0 ? p[0] : m4 == 1 ? p[1] : m4 == 2 ? p[2] : 0.0f;
      qo[2 * y] = (__bf16)mine;
      qo[2 * y + 1] = (__bf16)(mine * (F32 ? 8.0f : -16.0f));
    }
    rows[wave][S * G][lane] = __builtin_bit_cast(u32x4, qo);
    const float x = -lse * kLog2e;
    rows[wave][S * G + 1][lane] = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_mfma_f32_16x16x32_bf16(spread(terms(x), lane < 16), ones(lane < 16), f32x4{}, 0, 0, 0));
    const bool f = __any(!(fabsf(x) <= kFarLse));
    if (lane == 0) far[wave] = f;
  };

  load(begin + wave * KT);
  const Codes codes;
  const int first = first_row(a, it, begin) / 16 * 16;
  const bool once = it.rows - first <= 64;
#pragma unroll 1
  for (int base = begin; base < end; base += 4 * KT) {
    const int t0 = base + wave * KT;
    bf16x8 kc[NU][G];
    uint32_t kw[NU][G];
    bool here[NU];
    int see[NU];
    float acc[NU] = {};
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      here[u] = in[u];
      see[u] = first_row(a, it, min(t0 + 16 * u + col, it.t - 1));
#pragma unroll
      for (int g = 0; g < G; ++g) {
        kc[u][g] = codes.operand<F32>(code[u][g]);
        kw[u][g] = word[u][g];
      }
    }
    load(t0 + 4 * KT);
    const int all = first_row(a, it, min(t0 + KT, it.t) - 1), from = first_row(a, it, min(t0, it.t - 1));
#pragma unroll 1
    for (int c0 = first; c0 < it.rows; c0 += 64) {
      if (base == begin || !once) {
        if (c0 != first || base != begin) __syncthreads();
        prepare(c0 + 16 * wave);
        __syncthreads();
      }
#pragma unroll 1
      for (int x = 0; x < 4; ++x) {
        const int r0 = c0 + 16 * x;
        if (t0 >= end || r0 >= it.rows || r0 + 16 <= from) continue;
        bf16x8 q[S][G];
#pragma unroll
        for (int z = 0; z < S; ++z)
#pragma unroll
          for (int y = 0; y < G; ++y) q[z][y] = __builtin_bit_cast(bf16x8, rows[x][z * G + y][lane]);
        const bf16x8 qo = __builtin_bit_cast(bf16x8, rows[x][S * G][lane]);
        const f32x4 nl = __builtin_bit_cast(f32x4, rows[x][S * G + 1][lane]);
        const bool plain = !__builtin_amdgcn_readfirstlane(far[x]) && r0 >= all && r0 + 16 <= it.rows;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          union {
            uint32_t d[4];
            bf16x8 v;
          } wk = {{0, 0, 0, 0}};
#pragma unroll
          for (int y = 0; y < G; ++y) wk.d[y] = kw[u][y];
          f32x4 v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qo, wk.v, f32x4{}, 0, 0, 0);
#pragma unroll
          for (int y = 0; y < G; ++y) {
            f32x4 d = {};
#pragma unroll
            for (int z = 0; z < S; ++z) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[z][y], kc[u][y], d, 0, 0, 0);
            const float ks = __builtin_bit_cast(float, kw[u][y] & 0xffff0000u);
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
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const float w = add_xor32(add_xor16(acc[u]));
      const int key = t0 + 16 * u + col;
      if (m4 == 0 && key < end) write_weight(a, it, key, here[u] ? w : 0.0f);
    }
  }
}

constexpr int kPagedTokens = 32;  // a wave

template <int D>
void launch(int dtype, const WeighShape& sh, const WeighArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n_items * a.H);
  if (dtype == HF_F32) {
    if (sh.few) weights_few_kernel<RowsF32<D>, 1><<<grid, 256, 0, s>>>(a);
    else weights_rows_kernel<RowsF32<D>, 1, 4><<<grid, 256, 0, s>>>(a);
  } else {
    if (sh.few) weights_few_kernel<RowsBf16<D>, 2><<<grid, 256, 0, s>>>(a);
    else if (sh.keys == 256) weights_rows_kernel<RowsBf16<D>, 2, 4><<<grid, 256, 0, s>>>(a);
    else weights_rows_kernel<RowsBf16<D>, 1, 4><<<grid, 256, 0, s>>>(a);
  }
}

}  // namespace

WeighShape weigh_shape(int dtype, bool paged, int32_t B, const int32_t* q_len, const int32_t* kv_len, int32_t G,
                       int32_t H, int32_t d_h, int32_t causal) {
  WeighShape sh;
  sh.chunk = 0;
  sh.few = 1;
  if (paged) {
    // As many tiles a workgroup as leave four workgroups (what the registers admit) for each CU:
    // 64 decoded tokens over 4,096 keys each, of 32 / 8 heads, 47 us, with two 69, with one tile
    // each 61; one over 29,119 9.4 us, with two 11.2.
    int64_t tiles = 0;
    for (int b = 0; b < B; ++b) tiles += (kv_len[b] + 4 * kPagedTokens - 1) / (4 * kPagedTokens);
    sh.keys = (int32_t)(4 * kPagedTokens * std::clamp<int64_t>((tiles * H + 1023) / 1024, 1, 64));
    return sh;
  }
  int64_t longest = 0, keys = 0;
  for (int b = 0; b < B; ++b) {
    longest = std::max(longest, (int64_t)q_len[b] * G);
    keys += kv_len[b];
  }
  // Up to 32 query rows a head (fp32: 64) waves load them for themselves, more go through LDS.  us,
  // for itself / through LDS, bf16 heads of 128, 32 / 8 of them: 16 x 1 token over 4,096 keys 28 /
  // 35, 4 x 8 tokens 9.8 / 10.9, 4 x 16 12.5 / 10.3, 4 x 32 16.7 / 14.0; fp32, 16 / 4 heads of 128:
  // 4 x 8 15.7 / 20.9, 4 x 32 37 / 30; 14 / 2 heads of 64: 8 over 2,001 keys 7.0 / 7.2, 32 15.5 / 13.9.
  if (longest <= (dtype == HF_F32 ? 64 : 32)) {
    sh.keys = dtype == HF_F32 ? 128 : 256;
    return sh;
  }
  // Tiles of 256 keys (bf16) or 128, and the parts of the rows: the cut with the least time by
  // rounds of two workgroups a CU, of `start` and so much a stage (measured, us: one round of 8
  // stages of bf16 heads of 128 22, of fp32 heads of 64 34), and the join of the parts.  Tiles of
  // 128 keys alone: prompt of 8,192, 16 / 2 heads of 128, 234 us for 194; tiles of 256 alone: 1,024,
  // 32 / 8 heads of 64, 16.7 for 13.3.
  sh.few = 0;
  const bool f32 = dtype == HF_F32, wide = d_h == 128;
  double best = 1e30;
  for (int kb = f32 ? 1 : 2; kb >= 1; --kb) {
    const int tile = 128 * kb;
    const double stage = f32 ? (wide ? 11.0 : 5.7) : wide ? (kb == 2 ? 2.3 : 1.9) : (kb == 2 ? 1.4 : 1.0);
    const double start = 6.0;
    for (int64_t stages = 4;; stages += (stages + 3) / 4) {
      const int64_t chunk = 64 * stages;
      double items = 0;
      for (int b = 0; b < B; ++b) {
        const int64_t rows = (int64_t)q_len[b] * G, tiles = ((int64_t)kv_len[b] + tile - 1) / tile;
        const int64_t parts = std::max<int64_t>((rows + chunk - 1) / chunk, 1);
        const int64_t some = std::min<int64_t>(parts, 32);  // (of many parts, these, evenly)
        WeighSeq s = {};
        s.n = q_len[b];
        s.t = kv_len[b];
        s.tiles = (int32_t)tiles;
        s.parts = (int32_t)parts;
        double seen = 0;
        for (int64_t i = 0; i < some; ++i)
          seen += weigh_tiles(s, G, (int32_t)std::min<int64_t>(chunk, INT32_MAX), tile, causal, (int32_t)(parts * (2 * i + 1) / (2 * some)));
        items += seen / some * parts;
      }
      const double rounds = std::max(std::ceil(items * H / 512), 1.0);
      const double shared = items * H > 256 ? 1.0 : 0.55;
      const int64_t parts = std::max<int64_t>((longest + chunk - 1) / chunk, 1);
      const double us = rounds * (start + std::min(stages, (longest + 63) / 64) * stage * shared) +
                        (parts > 1 ? 5.0 + parts * keys * H * 8e-6 / 4 : 0.0);
      if (us < best) {
        best = us;
        sh.keys = tile;
        sh.chunk = parts > 1 ? (int32_t)chunk : 0;
      }
      if (parts <= 1) break;
    }
  }
  return sh;
}

int32_t weigh_parts(const WeighShape& sh, int64_t rows) {
  return sh.chunk ? (int32_t)std::max<int64_t>((rows + sh.chunk - 1) / sh.chunk, 1) : 1;
}

hipError_t launch_attention_weights(int dtype, int d_h, const WeighShape& sh, const WeighArgs& a, hipStream_t s) {
  if (d_h == 128)
    launch<128>(dtype, sh, a, s);
  else
    launch<64>(dtype, sh, a, s);
  hipError_t e = hipGetLastError();
  if (a.part && e == hipSuccess) {
    weights_join_kernel<<<(unsigned)(a.n_tiles * a.H), 256, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
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
