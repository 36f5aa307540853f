// Attention over dense keys and values: whole prompts, suffixes over a transferred
// cache, single tokens.
//
//   out_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i),  s_ij = scale <q_i, k_j>
//
// in one pass over the keys with a running maximum and sum (a row's sums are
// rescaled when its maximum is raised).  A wave owns a block of query rows and
// computes S^T = K Q^T, so that a lane holds scores of one row: the row's maximum
// and sum are sums over the lane's registers and one or two exchanges between
// lanes, and the weights, as they lie in the result registers, are the operand of
// the second product O^T = V^T P^T when V^T is read with its keys in the same
// order.  So weights never leave the registers.
//
// Keys and values stream through two LDS stages filled by global-to-LDS loads, the
// next tile's in flight while the current one is multiplied.
//
// Two kernel shapes; a call takes the faster one by their measured times (prompt_shape
// holds them, the call's planning compares):
//  - by rows: the waves of a workgroup share a tile of keys, each with query rows
//    of its own;
//  - by keys: the waves share the rows (one block) and deal the tiles of keys among
//    them, each with LDS stages of its own and no barrier in the loop; their
//    results are joined in LDS at the end.  For single tokens and short runs and
//    prompts, which the reading of the keys or the latency of a few tiles bounds.
// Where the workgroups are too few to fill the chip the key range is cut into parts
// as well, joined by attention_join_kernel.
#include <hip/hip_runtime.h>

#include "hf_attn.h"

namespace hf {
namespace {

// ---------------------------------------------------------------------------
// Operand layouts of one wave's tile: RW query rows against KT keys.
// ---------------------------------------------------------------------------

// The order of a block's LDS reads and matrix instructions: AHEAD of N steps of R reads
// each first, then one step's instruction and a later step's reads in turn.  Left to
// itself the compiler waits for most reads right after it issues them: prompts of 8,192
// tokens with heads of 128 519 us, with 4 steps ahead 505; of 5,000 with heads of 64 139,
// with 2 ahead 134 (with 4 139.5, for want of reads); fp32 prompts of 2,001 tokens with
// heads of 64 84.0, with 8 reads of values ahead 81.6.
template <int AHEAD, int R, int N>
FI void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * R, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// bf16 on v_mfma_f32_32x32x16_bf16: lane l is row l % 32; with h = l / 32, result
// register i of a 32-key block is key 8 (i / 4) + 4 h + i % 4, and of a 32-channel
// block the channel of that number.
template <int D_, int KT_>
struct Bf16Tile {
  static constexpr int D = D_, KT = KT_;
  static constexpr int RW = 32;
  static constexpr int NS = KT / 2, NO = D / 2;  // score and output registers
  static constexpr int ROWB = D * 2;             // bytes of a row
  static constexpr int AHEAD = D == 128 ? 4 : 2;
  typedef uint16_t T;
  struct Q {
    bf16x8 f[D / 16];
  };

  FI static int row(int lane) { return lane & 31; }
  FI static int key(int lane, int i) { return 32 * (i / 16) + 8 * ((i & 15) >> 2) + 4 * (lane >> 5) + (i & 3); }
  FI static int channel(int lane, int i) { return key(lane, i); }
  FI static float row_max(float x) { return max_xor32(x); }
  FI static float row_sum(float x) { return add_xor32(x); }

  // Where 16-byte chunk c of row r lies in a stage.  Keys are read 16 bytes a lane
  // by 32 rows at once, values 32 bytes of 8 rows at once (transposing reads); the
  // two exclusive-or orders put either on distinct banks.
  FI static int slot_k(int r, int c) { return c ^ (D == 128 ? r & 15 : (r >> 1) & 7); }
  FI static int slot_v(int r, int c) { return c ^ (2 * (D == 128 ? r & 7 : (r >> 1) & 3)); }

  FI static void load_q(Q& q, const T* row, int lane) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      q.f[c] = *reinterpret_cast<const bf16x8*>(row + 16 * c + 8 * (lane >> 5));
  }

  FI static void keep(Q& q) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) asm volatile("" : "+v"(q.f[c]));
  }

  FI static void scores(const Q& q, const unsigned char* sk, int lane, float (&s)[NS]) {
    const int r = lane & 31;
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb) {
      f32x16 acc = {};
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(
            sk + kb * 32 * ROWB + r * ROWB + slot_k(r, 2 * c + (lane >> 5)) * 16);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q.f[c], acc, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s[16 * kb + i] = acc[i];
    }
    reads_ahead<AHEAD, 1, KT / 32 * D / 16>();
  }

  typedef f32x16 O[D / 32];
  // O += V^T P^T.  CLEAN: values that are not finite enter as 0.
  template <bool CLEAN>
  FI static void values(O& o, const unsigned char* sv, int lane, const float (&p)[NS]) {
    // Weights of one bf16 rounding: in two terms, which would hold 16 bits, the product would
    // take twice its instructions, for an error that is the result's own rounding once more
    // (over prompts 2.1e-3 of the result's size in all against 1.7e-3 of the rounding alone).
    // The sum of the weights is of those before it.
    // The transposing read gives lane i of 16 the values of 4 rows at channel i; its
    // lane i names row i / 4 of them and 8 bytes there
    const int h = lane >> 5, gb = (lane >> 4) & 1, i = lane & 15;
    const int r = 4 * h + (i >> 2);
#pragma unroll
    for (int c = 0; c < KT / 16; ++c) {
      union {
        bf16x8 v;
        uint32_t u[4];
      } b;
#pragma unroll
      for (int y = 0; y < 4; ++y) b.u[y] = pack_bf16(p[8 * c + 2 * y], p[8 * c + 2 * y + 1]);
#pragma unroll
      for (int n = 0; n < D / 32; ++n) {
        const unsigned char* at = sv + (16 * c + r) * ROWB + slot_v(r, 4 * n + 2 * gb) * 16 + (i & 3) * 8;
        union {
          bf16x8 v;
          s16x4 s[2];
          uint32_t u[4];
        } a;
        a.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)at);
        a.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 8 * ROWB));
        if (CLEAN) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            if ((a.u[y] & 0x7f80u) == 0x7f80u) a.u[y] &= 0xffff0000u;
            if ((a.u[y] & 0x7f800000u) == 0x7f800000u) a.u[y] &= 0xffffu;
          }
        }
        o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, o[n], 0, 0, 0);
      }
    }
    if (!CLEAN) reads_ahead<AHEAD, 2, KT / 16 * D / 32>();
  }

  FI static float value_at(const unsigned char* sv, int r, int ch) {
    const uint16_t x = *reinterpret_cast<const uint16_t*>(sv + r * ROWB + slot_v(r, ch >> 3) * 16 + (ch & 7) * 2);
    return __builtin_bit_cast(float, (uint32_t)x << 16);
  }
  FI static float get(const O& o, int i) { return o[i / 16][i & 15]; }
  FI static void set(O& o, int i, float x) { o[i / 16][i & 15] = x; }
  FI static void store4(T* p, const float (&x)[4]) {
    const u32x2 v = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    *reinterpret_cast<u32x2*>(p) = v;
  }
};

// fp32 on v_mfma_f32_16x16x4_f32: lane l is row l % 16; with m = l / 16, result
// register i of a 16-key (16-channel) block is key (channel) 4 m + i.  Step (u, j)
// of the first product takes channel 16 u + 4 m + j, so that a lane's operands are
// 16-byte loads; step i of the second takes key 4 m + i, so that the scores'
// registers are its operands as they are.
template <int D_, int KT_>
struct F32Tile {
  static constexpr int D = D_, KT = KT_;
  static constexpr int RW = 16;
  static constexpr int NS = KT / 4, NO = D / 4;
  static constexpr int ROWB = D * 4;
  typedef float T;
  struct Q {
    f32x4 f[D / 16];
  };

  FI static int row(int lane) { return lane & 15; }
  FI static int key(int lane, int i) { return 16 * (i / 4) + 4 * (lane >> 4) + (i & 3); }
  FI static int channel(int lane, int i) { return key(lane, i); }
  FI static float row_max(float x) { return max_xor32(max_xor16(x)); }
  FI static float row_sum(float x) { return add_xor32(add_xor16(x)); }

  FI static int slot_k(int r, int c) { return c ^ (r & 15); }
  FI static int slot_v(int r, int c) { return c ^ (((r >> 2) & 3) << 2); }

  FI static void load_q(Q& q, const T* row, int lane) {
#pragma unroll
    for (int u = 0; u < D / 16; ++u)
      q.f[u] = *reinterpret_cast<const f32x4*>(row + 16 * u + 4 * (lane >> 4));
  }

  FI static void keep(Q& q) {
#pragma unroll
    for (int u = 0; u < D / 16; ++u) asm volatile("" : "+v"(q.f[u]));
  }

  FI static void scores(const Q& q, const unsigned char* sk, int lane, float (&s)[NS]) {
    const int r = lane & 15;
#pragma unroll
    for (int kb = 0; kb < KT / 16; ++kb) {
      f32x4 acc = {};
#pragma unroll
      for (int u = 0; u < D / 16; ++u) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(
            sk + (kb * 16 + r) * ROWB + slot_k(r, 4 * u + (lane >> 4)) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], q.f[u][j], acc, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * kb + i] = acc[i];
    }
  }

  typedef f32x4 O[D / 16];
  template <bool CLEAN>
  FI static void values(O& o, const unsigned char* sv, int lane, const float (&p)[NS]) {
    const int m = lane >> 4, c = lane & 15;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      const int r = 16 * (k / 4) + 4 * m + (k & 3);
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        float a = *reinterpret_cast<const float*>(sv + r * ROWB + slot_v(r, 4 * n + (c >> 2)) * 16 + (c & 3) * 4);
        if (CLEAN) a = finite_bits(a) ? a : 0.0f;
        o[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, p[k], o[n], 0, 0, 0);
      }
    }
    if (!CLEAN) reads_ahead<8, 1, NS * D / 16>();
  }

  FI static float value_at(const unsigned char* sv, int r, int ch) {
    return *reinterpret_cast<const float*>(sv + r * ROWB + slot_v(r, ch >> 2) * 16 + (ch & 3) * 4);
  }
  FI static float get(const O& o, int i) { return o[i / 4][i & 3]; }
  FI static void set(O& o, int i, float x) { o[i / 4][i & 3] = x; }
  FI static void store4(T* p, const float (&x)[4]) {
    const f32x4 v = {x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p) = v;
  }
};

// ---------------------------------------------------------------------------
// One tile of keys against a wave's rows.
// ---------------------------------------------------------------------------
template <class P>
struct Rows {
  typename P::Q q;
  typename P::O o;
  float m, l;  // the row's maximum; this lane's share of its weight
  bool far;    // m is in units of far_unit(c), not of c (second pass)
  int last;    // the last key it sees
};

// The weights of a tile's scores and their product with its values.  MASK: some row
// of the wave may not see every key of the tile (t0 is its first); edge: there is one.
// In such a tile a value that is not finite would reach rows that do not see it, as
// 0 * NaN.  That shows in their results: the kernels look at them at the end and in
// that case compute once more with `careful`, where such a value enters the product
// as 0 and is added to the rows that see its key.  (In other tiles all rows see all
// keys, and the product does what it should.)  The second pass, whose tiles are all taken
// with MASK, also gives each row the unit that its scores need.
template <class P, bool MASK>
FI void finish(Rows<P>& w, float (&s)[P::NS], const unsigned char* sv, int lane, float c, int t0,
               bool careful, bool edge) {
  float cr = MASK && w.far ? far_unit(c) : c;
  if (MASK) {
#pragma unroll
    for (int i = 0; i < P::NS; ++i)
      if (t0 + P::key(lane, i) > w.last) s[i] = -INFINITY;
  }
  float mx = s[0];
#pragma unroll
  for (int i = 1; i < P::NS; ++i) mx = fmaxf(mx, s[i]);
  mx = P::row_max(mx);
  if (__any(mx * cr > w.m + kRaise)) {
    const float f = raise(mx, c, MASK && careful, cr, w.m);  // (each row by its own scores alone)
    if (MASK) w.far = cr != c;
    w.l *= f;
#pragma unroll
    for (int i = 0; i < P::NO; ++i) P::set(w.o, i, P::get(w.o, i) * f);
  }
#pragma unroll
  for (int i = 0; i < P::NS; ++i) {
    s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], cr, -w.m));
    w.l += s[i];
  }
  if (!MASK || !careful || !edge) {
    P::template values<false>(w.o, sv, lane, s);
    return;
  }
  P::template values<true>(w.o, sv, lane, s);
  for (int r = 0; r < P::KT && t0 + r <= w.last; ++r) {
    int at = lane;  // (opaque: the addresses below are formed here, not kept across the kernel)
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int i = 0; i < P::NO; ++i) {
      const float v = P::value_at(sv, r, P::channel(at, i));
      if (!finite_bits(v)) P::set(w.o, i, P::get(w.o, i) + v);
    }
  }
}

// Whether a row is to be computed a second time.  saw: it saw a key.
template <class P>
FI bool second_pass(const Rows<P>& w, bool saw) {
  bool bad = saw && far_max(w.m);
#pragma unroll
  for (int i = 0; i < P::NO; ++i) bad |= !finite_bits(P::get(w.o, i));
  return bad;
}

// Loads of one tile (keys t0 .. t0 + KT) into a stage: NB of the tile's 1 KB blocks
// from block b0 in steps of `bstep`.  The tile's address is in scalar registers, a lane's
// place in the tile a 32-bit offset (rows lie at most 2^23 elements apart: host check).
// The buffer ends with the last key: rows past it are not read (what their place in the
// stage holds is masked), and no lane compares.
// UNSEEN: as instructions that the compiler does not see as LDS accesses.  By keys it
// would wait for all loads before it reads a stage, the next tile's in flight among
// them; the kernel's own waits are what there has to be.
template <class P, bool V, int NB, bool UNSEEN>
struct Fetch {
  typedef typename P::T T;
  static constexpr int CPR = P::ROWB / 16;  // chunks a row
  static_assert(P::KT * (1ll << 23) * sizeof(T) <= 1ll << 31, "32-bit offsets");
  const char* base;
  long long st;  // bytes
  int t;
  int off[NB];

  FI static int row(int i, int b0, int bstep, int lane) { return (b0 + i * bstep) * (64 / CPR) + lane / CPR; }
  FI static int chunk(int r, int lane) {  // (its own inverse)
    return (V ? P::slot_v(r, lane % CPR) : P::slot_k(r, lane % CPR)) * 16;
  }
  FI void init(const T* base_, long long st_, int t_, int b0, int bstep, int lane) {
    base = reinterpret_cast<const char*>(base_);
    st = st_ * (int)sizeof(T);
    t = t_;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int r = row(i, b0, bstep, lane);
      off[i] = r * (int)st + chunk(r, lane);
    }
  }
  FI void get(int t0, unsigned char* stage, int b0, int bstep) const {
    const char* tile = base + t0 * st;
    const int bytes = (int)min((t - 1 - t0) * st + P::ROWB, (long long)INT32_MAX);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      unsigned char* to = stage + (b0 + i * bstep) * 1024;
      if (UNSEEN)
        load_lds_unseen(tile, bytes, off[i], to);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer_at(tile, bytes), (lds_void_t*)to, 16, off[i], 0, 0, 0);
    }
  }
};

// The part of row r.
template <class P>
FI void write_part(const AttnIO& io, const AttnItem& it, int r, float m, float l, const typename P::O& o,
                   int lane) {
  const long long slot = part_slot(it, r);
  float* po = io.part + slot * P::D;
#pragma unroll
  for (int i = 0; i < P::NO; i += 4) {
    const f32x4 v = {P::get(o, i), P::get(o, i + 1), P::get(o, i + 2), P::get(o, i + 3)};
    *reinterpret_cast<f32x4*>(po + P::channel(lane, i)) = v;
  }
  if (lane < P::RW) {
    io.ml[2 * slot] = m;
    io.ml[2 * slot + 1] = l;
  }
}

// The results of a wave's finished rows.  In bf16 through RW rows of LDS of its own: a
// lane holds four channels of its row, 8 bytes, and written from there an instruction
// would touch 32 rows (a packed batch of six prompts 241 and like this 236 us; 256 queries
// over 300 keys each 47.8 and 43.9).  In fp32 an instruction writes 64 bytes of a row
// anyway, and the detour costs 2%.
// 16-byte chunk c of row r lies at c ^ (r % 16) (r % 8 in rows of 8 chunks).
template <class P>
FI void write_rows(const AttnIO& io, const AttnSeqs& s, const AttnItem& it, int row0, float m, float l,
                   const typename P::O& o, unsigned char* lds, int lane) {
  typedef typename P::T T;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int CPR = P::ROWB / 16, EPC = 16 / sizeof(T);
  auto slot = [](int r, int c) { return r * P::ROWB + (c ^ (r & (CPR < 16 ? CPR - 1 : 15))) * 16; };
  auto place = [&](int r) {
    const int token = divide(r, s.by_g), head = it.h * s.G + r - token * s.G;
    return static_cast<T*>(io.out) + out_at(io, s, it, token, head);
  };
  const int mine = P::row(lane);
  const bool on = row0 + mine < it.rows;
  const float inv = inverse_weight(m, l);
  T* out = F32 && on ? place(row0 + mine) : nullptr;
#pragma unroll
  for (int i = 0; i < P::NO; i += 4) {
    const int ch = P::channel(lane, i);
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = P::get(o, i + j) * inv;
    if (!F32)
      P::store4(reinterpret_cast<T*>(lds + slot(mine, ch / EPC)) + ch % EPC, x);
    else if (on)
      P::store4(out + ch, x);
  }
  if (lane < P::RW && on) {
    const int token = divide(row0 + mine, s.by_g), head = it.h * s.G + row0 + mine - token * s.G;
    write_lse(io, s, it, token, head, m, l);
  }
  if (F32) return;
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < P::RW * CPR / 64; ++i) {
    const int rl = i * (64 / CPR) + lane / CPR, c = lane % CPR;
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + slot(rl, c));
    if (row0 + rl < it.rows) *reinterpret_cast<u32x4*>(place(row0 + rl) + c * EPC) = v;
  }
}

// Row r (the last one for rows past it, which are not written).
template <class P>
FI void load_row(Rows<P>& w, const AttnArgs& a, const AttnItem& it, int r, int lane) {
  typedef typename P::T T;
  const AttnSeqs& s = a.s;
  r = min(r, it.rows - 1);
  const int token = divide(r, s.by_g), head = it.h * s.G + r - token * s.G;
  P::load_q(w.q, static_cast<const T*>(a.io.q) + seq_at(it.b, it.row0, a.io.q_sb, a.io.q_st) +
                     token * a.io.q_st + head * a.io.q_sh, lane);
  w.last = last_key(s, it, token);
}
template <class P>
FI void clear_row(Rows<P>& w, bool careful) {
#pragma unroll
  for (int i = 0; i < P::NO; ++i) P::set(w.o, i, 0.0f);
  w.m = kNoMax;
  w.l = 0.0f;
  w.far = careful;
}

template <bool M>
struct Flag {
  static constexpr bool value = M;
};

// By rows: NW waves, each with RW rows of the tile, all against the same keys.  A wave
// computes the scores of the next tile before it finishes this one's, so
// that matrix instructions and the softmax's are there to be issued side by side.
// Bound by the matrix cores and the softmax's instructions beside them: causal prompts of
// 32 heads of 128 on 8, 8,192 tokens in 475 to 515 us, by card (1.07 to 1.16 PFLOP/s; a large
// library product, 16384^3, reaches 1.37); 14 fp32 heads of 64, 2,001 tokens, in 81 (88
// TFLOP/s: the longest tile has a CU almost to itself and takes all of it, 2,001 keys at 37 ns
// and 5.8 us of start; 3,000 tokens of 32 heads of 128 reach 127 of the 153 that a library
// product does).
// Eight waves and one workgroup a CU in bf16: with 64 rows a wave the registers spill (777
// against 540 us for 8,192 tokens), with four waves and two workgroups a CU the tiles are
// loaded twice (701 against 588), and waves started half a tile apart, given
// priority in turn or held back between the products gained nothing (600, 568, 565 against
// 540).  In fp32 four waves and up to four workgroups a CU (with heads of 64; two with 128).
template <class P, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attention_rows_kernel(const AttnArgs a) {
  typedef typename P::T T;
  constexpr int KT = P::KT, WR = P::RW;  // keys a tile, rows a wave
  __shared__ __attribute__((aligned(1024))) unsigned char k0[KT * P::ROWB];
  __shared__ __attribute__((aligned(1024))) unsigned char v0[KT * P::ROWB];
  __shared__ __attribute__((aligned(1024))) unsigned char k1[KT * P::ROWB];
  __shared__ __attribute__((aligned(1024))) unsigned char v1[KT * P::ROWB];
  constexpr int NB = KT * P::ROWB / 1024 / NW;
  static_assert(NB * NW * 1024 == KT * P::ROWB, "whole blocks a wave");

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AttnSeqs& s = a.s;
  const AttnItem it = attn_item(s, NW * WR);
  const int t = it.t, n_rows = it.rows;
  const int row0 = it.tile * NW * WR, my0 = row0 + wave * WR;
  Rows<P> w;

  // keys of this part that some row of the workgroup sees, and that all of them see
  const int wg_last = last_key(s, it, divide(min(row0 + NW * WR - 1, n_rows - 1), s.by_g));
  const int wg_first = last_key(s, it, divide(row0, s.by_g));
  const int wave_last = last_key(s, it, divide(min(my0 + WR - 1, n_rows - 1), s.by_g));
  const int lo = it.part * s.chunk;
  const int hi = min(wg_last + 1, it.parts == 1 ? t : min(t, lo + s.chunk));
  const T* kb = static_cast<const T*>(a.k) + seq_at(it.b, it.key0, a.k_sb, a.k_st) + (long long)it.h * a.k_sh;
  const T* vb = static_cast<const T*>(a.v) + seq_at(it.b, it.key0, a.v_sb, a.v_st) + (long long)it.h * a.v_sh;
  const float c = a.io.c;

  Fetch<P, false, NB, false> fk;
  Fetch<P, true, NB, false> fv;
  fk.init(kb, a.k_st, t, wave, NW, lane);
  fv.init(vb, a.v_st, t, wave, NW, lane);
  // nothing past the range's last tile is loaded, or used
  auto get_k = [&](int t0, unsigned char* st) {
    if (t0 < hi) fk.get(t0, st, wave, NW);
  };
  auto get_v = [&](int t0, unsigned char* st) {
    if (t0 < hi) fv.get(t0, st, wave, NW);
  };
  auto ready = [&]() {  // every wave's loads are there, and no wave reads what is loaded next
    __builtin_amdgcn_s_waitcnt(kWaitMemory);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  typedef float Scores[P::NS];
  // Tile t0, whose scores are in s, with its values in sv; the next tile's keys in nk.
  auto step = [&](int t0, Scores& s0, Scores& s1, unsigned char* sk, unsigned char* sv,
                  unsigned char* nk, unsigned char* nv) {
    ready();
    get_k(t0 + 2 * KT, sk);
    get_v(t0 + KT, nv);
    P::scores(w.q, nk, lane, s1);
    finish<P, false>(w, s0, sv, lane, c, t0, false, false);
  };
  bool careful = false;
  // Near a causal edge or the last key, one tile's scores at a time.
  auto masked_step = [&](int t0, Scores& s, unsigned char* sk, unsigned char* sv,
                         unsigned char* nk, unsigned char* nv) {
    ready();
    get_k(t0 + 2 * KT, sk);
    get_v(t0 + KT, nv);
    if (t0 <= wave_last) finish<P, true>(w, s, sv, lane, c, t0, careful, t0 + KT - 1 > wg_first);
    if (t0 + KT <= wave_last && t0 + KT < hi) P::scores(w.q, nk, lane, s);
  };
  // what the first two steps need is on its way at once
  auto get_first = [&]() {
    get_k(lo, k0);
    get_v(lo, v0);
    get_k(lo + KT, k1);
  };
  get_first();
  load_row<P>(w, a, it, my0 + P::row(lane), lane);
  for (;;) {
    clear_row<P>(w, careful);
    if (lo < hi) {
      Scores s0, s1;
      if (careful) get_first();
      ready();
      P::scores(w.q, k0, lane, s0);
      // pairs of tiles that every row sees whole, with a tile after them
      int t0 = lo;
      for (; !careful && t0 + 2 * KT - 1 <= wg_first && t0 + 2 * KT < hi; t0 += 2 * KT) {
        step(t0, s0, s1, k0, v0, k1, v1);
        step(t0 + KT, s1, s0, k1, v1, k0, v0);
      }
      for (; t0 < hi; t0 += 2 * KT) {
        masked_step(t0, s0, k0, v0, k1, v1);
        if (t0 + KT < hi) masked_step(t0 + KT, s0, k1, v1, k0, v0);
      }
    }
    // a barrier in both passes: after it no wave reads keys or values of this pass
    const bool again = __syncthreads_or(second_pass(w, lo < hi && lo <= w.last));
    if (careful || !again) break;
    careful = true;
  }
  const float l = P::row_sum(w.l);
  if (careful) w.m = end_max(w.m, w.far ? far_unit(c) : c, c, l, lo < hi && lo <= w.last);
  if (it.parts > 1) {
    const int r = my0 + P::row(lane);
    if (r < n_rows) write_part<P>(a.io, it, r, w.m, l, w.o, lane);
    return;
  }
  // (no wave reads keys or values any more: both passes end with a barrier)
  static_assert(NW % 4 == 0 && NW / 4 * WR * P::ROWB <= KT * P::ROWB, "rows in the stages");
  unsigned char* mine = (wave & 3) == 0 ? k0 : (wave & 3) == 1 ? v0 : (wave & 3) == 2 ? k1 : v1;
  write_rows<P>(a.io, s, it, my0, w.m, l, w.o, mine + wave / 4 * WR * P::ROWB, lane);
}

// By keys: one block of RW rows, the tiles of keys dealt to NW waves.  Bound by HBM for
// one block of rows: a token of 32 heads on 8 of 128 over 29K keys 23 us (5.2 TB/s), four
// over 12K keys together 14.7 and 4.0 us for the join; for few keys by the latency of the
// loads that follow each other (8.6 us for a prompt of 100 tokens).  Tiles of 32 keys: two
// stages of four waves fill 128 KB of LDS (fp32 rows of 128 channels are twice as long, and
// take 16).
template <class P, int NW>
__global__ __launch_bounds__(NW * 64) void attention_keys_kernel(const AttnArgs a) {
  typedef typename P::T T;
  constexpr int TB = P::KT * P::ROWB;  // bytes of a tile of keys, or of values
  __shared__ __attribute__((aligned(1024))) unsigned char s0[NW * 2 * TB];
  __shared__ __attribute__((aligned(1024))) unsigned char s1[NW * 2 * TB];
  __shared__ float sm[NW][P::RW], sl[NW][P::RW];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AttnSeqs& s = a.s;
  const AttnItem it = attn_item(s, P::RW);
  const int t = it.t, n_rows = it.rows;
  const int row0 = it.tile * P::RW;
  const int first = last_key(s, it, divide(min(row0, n_rows - 1), s.by_g));
  const int last = last_key(s, it, divide(min(row0 + P::RW - 1, n_rows - 1), s.by_g));
  const int lo = it.part * s.chunk + wave * P::KT;
  const int hi = min(last + 1, it.parts == 1 ? t : min(t, it.part * s.chunk + s.chunk));
  const T* kb = static_cast<const T*>(a.k) + seq_at(it.b, it.key0, a.k_sb, a.k_st) + (long long)it.h * a.k_sh;
  const T* vb = static_cast<const T*>(a.v) + seq_at(it.b, it.key0, a.v_sb, a.v_st) + (long long)it.h * a.v_sh;
  const float c = a.io.c;
  unsigned char* w0 = s0 + wave * 2 * TB;
  unsigned char* w1 = s1 + wave * 2 * TB;

  Fetch<P, false, TB / 1024, true> fk;
  Fetch<P, true, TB / 1024, true> fv;
  fk.init(kb, a.k_st, t, 0, 1, lane);
  fv.init(vb, a.v_st, t, 0, 1, lane);
  auto get = [&](int t0, unsigned char* st) {
    fk.get(t0, st, 0, 1);
    fv.get(t0, st + TB, 0, 1);
  };
  Rows<P> w;
  bool careful = false;
  // Waits until at most n loads after those of the tile at hand are outstanding.
  constexpr int NL = TB / 1024;  // loads of a tile's keys, or values
  auto ready = [&](bool next, auto values) {
    constexpr int n = decltype(values)::value ? 0 : NL;
    if (next)
      __builtin_amdgcn_s_waitcnt(wait_vm_only(n + 2 * NL));
    else
      __builtin_amdgcn_s_waitcnt(wait_vm_only(n));
    asm volatile("" ::: "memory");
  };
  auto step = [&](int t0, unsigned char* st, unsigned char* nst) {
    const bool next = t0 + NW * P::KT < hi;
    __builtin_amdgcn_s_waitcnt(kWaitLds);  // (what was read of nst is in registers)
    if (next) get(t0 + NW * P::KT, nst);
    ready(next, Flag<false>());
    float s[P::NS];
    P::scores(w.q, st, lane, s);
    ready(next, Flag<true>());
    const bool edge = t0 + P::KT - 1 > first;
    if (careful || edge)
      finish<P, true>(w, s, st + TB, lane, c, t0, careful, edge);
    else
      finish<P, false>(w, s, st + TB, lane, c, t0, false, false);
  };
  // The first tile on its way, then the queries; both are waited for here, for a wait for
  // the queries inside the loop would wait for the tiles in flight as well.
  if (lo < hi) get(lo, w0);
  load_row<P>(w, a, it, row0 + P::row(lane), lane);
  P::keep(w.q);
  for (;;) {
    clear_row<P>(w, careful);
    if (lo < hi) {
      if (careful) get(lo, w0);
      for (int t0 = lo; t0 < hi; t0 += 2 * NW * P::KT) {
        step(t0, w0, w1);
        if (t0 + NW * P::KT < hi) step(t0 + NW * P::KT, w1, w0);
      }
    }
    if (careful || !__any(second_pass(w, lo < hi && lo <= w.last))) break;
    careful = true;
  }

  const int rl = P::row(lane);
  const float l = P::row_sum(w.l);
  if (careful) w.m = end_max(w.m, w.far ? far_unit(c) : c, c, l, lo < hi && lo <= w.last);
  if (lane < P::RW) {
    sm[wave][rl] = w.m;
    sl[wave][rl] = l;
  }
  __syncthreads();
  float m = kNoMax;
#pragma unroll
  for (int x = 0; x < NW; ++x) m = fmaxf(m, sm[x][rl]);
  const float f = __builtin_amdgcn_exp2f(w.m - m);
  f32x4* sums = reinterpret_cast<f32x4*>(s0);
  static_assert(NW * P::RW * P::D * 4 <= NW * 2 * TB, "joining buffer");
#pragma unroll
  for (int i = 0; i < P::NO; i += 4) {
    const f32x4 v = {P::get(w.o, i), P::get(w.o, i + 1), P::get(w.o, i + 2), P::get(w.o, i + 3)};
    sums[sum_slot<P::RW, P::D>(wave, rl, P::channel(lane, i) / 4)] = v * f;
  }
  __syncthreads();
  write_joined<P::RW, P::D, NW, sizeof(T) == 4>(a.io, s, it, row0, sums, sm, sl);
}

// ---------------------------------------------------------------------------
// The parts of split rows: out = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p.
// A row has D / 4 threads of four channels for every SL-th part, so that its parts are
// loaded at the same time: one wave a row, part after part, took 19 us for 57 parts of
// 40 rows, this takes 4.9.  Bound by a launch's time with few rows, by the parts' bytes with
// many (31 MB in 9.5 us).
// ---------------------------------------------------------------------------
struct JoinArgs {
  AttnIO io;
  AttnSeqs s;
};

template <bool F32, int D, int SL>
__global__ __launch_bounds__(256) void attention_join_kernel(const JoinArgs a) {
  constexpr int TC = D / 4, NR = 256 / (TC * SL);
  __shared__ f32x4 so[NR][SL][TC];
  __shared__ float sm[NR][SL], sl[NR][SL];
  const AttnSeqs& s = a.s;
  const int c = threadIdx.x % TC, q = threadIdx.x / TC % SL, rr = threadIdx.x / (TC * SL);
  int i = blockIdx.x * NR + rr;
  const bool on = i < s.n_split;
  static_assert(TC * SL >= 64, "a wave has one row");
  AttnItem it;
  it.b = find_seq(s.q, &AttnSeq::split0, s.B, __builtin_amdgcn_readfirstlane(i));
  const AttnSeq sq = s.q[it.b];
  it.row0 = sq.row0;
  i -= sq.split0;
  const int parts = on ? sq.parts : 0;
  const long long slot = sq.part0 + (long long)i * parts;
  const float* ml = a.io.ml + 2 * slot;
  const float* po = a.io.part + slot * D + 4 * c;
  float m = kNoMax, least = kNoMax, l = 0.0f;
  f32x4 o = {};
#pragma unroll 4
  for (int p = q; p < parts; p += SL) {
    m = fmaxf(m, ml[2 * p]);
    least = fminf(least, ml[2 * p]);
  }
#pragma unroll 4
  for (int p = q; p < parts; p += SL) {
    const float f = __builtin_amdgcn_exp2f(ml[2 * p] - m);
    const f32x4 v = *reinterpret_cast<const f32x4*>(po + (long long)p * D);
    l = fmaf(ml[2 * p + 1], f, l);
    o += v * f;
  }
  so[rr][q][c] = o;
  if (c == 0) {
    sm[rr][q] = l == 0.0f ? least : m;
    sl[rr][q] = l;
  }
  __syncthreads();
  if (q != 0 || !on) return;
  for (int x = 0; x < SL; ++x) {
    m = fmaxf(m, sm[rr][x]);
    least = fminf(least, sm[rr][x]);
  }
  o = f32x4{};
  l = 0.0f;
  for (int x = 0; x < SL; ++x) {
    const float f = __builtin_amdgcn_exp2f(sm[rr][x] - m);
    o += so[rr][x][c] * f;
    l = fmaf(sl[rr][x], f, l);
  }
  if (l == 0.0f) m = least;
  const int n_rows = sq.n * s.G, h = i / n_rows, r = i - h * n_rows;
  const int token = divide(r, s.by_g), head = h * s.G + r - token * s.G;
  const long long at = out_at(a.io, s, it, token, head) + 4 * c;
  o *= inverse_weight(m, l);
  if (F32) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.io.out) + at) = o;
  } else {
    const u32x2 v = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.io.out) + at) = v;
  }
  if (c == 0) write_lse(a.io, s, it, token, head, m, l);
}

constexpr int kRowWaves = 8, kRowWavesF32 = 4, kKeyWaves = 4;

template <int D>
hipError_t launch(int dtype, const AttnShape& sh, const AttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.s.n_items * a.s.H));
  if (dtype == HF_BF16) {
    if (sh.by_keys)
      attention_keys_kernel<Bf16Tile<D, 32>, kKeyWaves><<<grid, kKeyWaves * 64, 0, st>>>(a);
    else
      attention_rows_kernel<Bf16Tile<D, 64>, kRowWaves><<<grid, kRowWaves * 64, 0, st>>>(a);
  } else {
    if (sh.by_keys)
      attention_keys_kernel<F32Tile<D, D == 128 ? 16 : 32>, kKeyWaves>
          <<<grid, kKeyWaves * 64, 0, st>>>(a);
    else  // (tiles of 64 keys: 91 us against 94 with heads of 64, 745 against 662 with 128)
      attention_rows_kernel<F32Tile<D, 32>, kRowWavesF32><<<grid, kRowWavesF32 * 64, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <bool F32, int D, int SL>
void join_by(const JoinArgs& a, hipStream_t st) {
  constexpr int NR = 256 / (D / 4 * SL);
  attention_join_kernel<F32, D, SL><<<(unsigned)((a.s.n_split + NR - 1) / NR), 256, 0, st>>>(a);
}
// With few rows eight threads of a channel share its parts, with many, which fill the chip
// anyway, as few as make a wave a row's.  Measured with eight and with two, us, d_h 128: 40
// rows of 57 parts 4.9 and 7.0, 448 rows of 17 parts 3.9 and 4.4; 5,120 rows of 4 parts 7.5
// and 5.4, 10,240 of 6 parts 10.7 and 9.5.
template <bool F32, int D>
void join(const JoinArgs& a, hipStream_t st) {
  if (a.s.n_split < 1024)
    join_by<F32, D, 8>(a, st);
  else
    join_by<F32, D, 256 / D>(a, st);
}

}  // namespace

// Times as the rule weighs them, d_h 128 and 64, with every workgroup on a CU of its own:
// parts of 64 to 1,024 keys by rows, of 128 to 4,096 by keys (keys from L2; where HBM bounds
// it, one tile of rows over 29K keys, 20 ns a key).  They were measured when the kernels took 5
// to 30% longer; now, us of start and ns a key by rows and by keys: bf16 of 128 11.2 + 26.6
// and 7.3 + 9.4, of 64 8.7 + 15.9 and 5.0 + 5.5; fp32 of 128 7.2 + 68.5 and 5.8 + 30.7, of 64
// 5.8 + 37.3 and 4.9 + 12.7.  What decides is how the two stand to each other, which has stayed
// the same within a fifth.  Parts for one workgroup a CU: for two, by
// keys with heads of 64, which LDS has room for, 18.9 us against 15.7 for a token over 29K.
// fp32 tiles by rows share a CU, up to four with heads of 64 and two with 128 (three is what
// the rule counts): a causal prompt's deal turns every other round (2,001 tokens with heads
// of 64: 113 us without, 95 with).
AttnShape prompt_shape(int dtype, int d_h, bool by_keys) {
  AttnShape sh;
  const bool f32 = dtype == HF_F32, wide = d_h == 128;
  const int rw = f32 ? 16 : 32;
  sh.by_keys = by_keys;
  sh.rows = by_keys ? rw : rw * (f32 ? kRowWavesF32 : kRowWaves);
  sh.wg_target = 256;
  sh.step = by_keys ? 32 * kKeyWaves : 64;
  sh.resident = by_keys || !f32 ? 1 : 3;
  if (by_keys) {
    sh.ns_start = f32 || !wide ? 6000 : 9600;
    sh.ns_key = f32 ? (wide ? 32 : 14) : wide ? 12 : 7;
  } else {
    sh.ns_start = f32 ? (wide ? 8000 : 6400) : wide ? 12000 : 10500;
    sh.ns_key = f32 ? (wide ? 80 : 44) : wide ? 30 : 17;
  }
  return sh;
}

hipError_t launch_prompt_attention(int dtype, int d_h, const AttnShape& sh, const AttnArgs& a,
                                   hipStream_t s) {
  return d_h == 128 ? launch<128>(dtype, sh, a, s) : launch<64>(dtype, sh, a, s);
}

hipError_t launch_attention_join(int dtype, int d_h, const AttnIO& io, const AttnSeqs& s,
                                 hipStream_t st) {
  JoinArgs a{io, s};
  if (dtype == HF_F32)
    d_h == 128 ? join<true, 128>(a, st) : join<true, 64>(a, st);
  else
    d_h == 128 ? join<false, 128>(a, st) : join<false, 64>(a, st);
  return hipGetLastError();
}

}  // namespace hf
