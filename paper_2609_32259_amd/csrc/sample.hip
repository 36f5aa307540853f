// The next token of each row of logits (hf_sample_tokens).
//
// With w_j = exp((x_j - max x) / T), and the tokens in falling order of w (equal ones by
// number), what stays under top-k, top-p and min-p is a prefix of that order, and the token
// is where the running sum of w passes u times the prefix's.  No sort is needed for that: the
// row is counted into bins of 1/128 in log w, which gives counts and sums up to every bin
// border, and only the bins in which one of the borders or the draw falls are looked at
// token by token.
//
// Sums.  A border decides a token, so that sums hold more than 32 bits.  A bin adds up the
// tokens' shortfalls 1 - exp(-f / 128) below the bin's upper edge (f: the place in the bin)
// as whole numbers of 2^-30, which fp32 forms to 2^-30: with the count that is the bin's sum
// of w to 2^-29 of itself, in whatever order the tokens come.  The bins reach down to
// exp(-32); what lies below has in all less than 2^20 exp(-32) = 2^-26 of the largest w and
// cannot be drawn (u < 1 - 2^-25).  Everything after the bins is in 64 bits.
#include <hip/hip_runtime.h>

#include "hf_attn.h"

namespace hf {
namespace {

constexpr int kBins = 4096;  // of 1/128 each
constexpr int kNT = 1024;    // threads of a row
constexpr int kBPT = kBins / kNT;
constexpr int kList = 2048;  // tokens that are put in order at a time
constexpr int kFew = 512;    // of top-k: half the threads, whose maxima bound it
constexpr int kFracBits = 43;  // shortfalls below, the count above

FI uint32_t ordered(float x) {  // whole numbers of the same order
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
FI float unordered(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// Place of a token in the falling order as one number: larger comes first.
FI uint64_t place(float x, int i) { return ((uint64_t)ordered(x) << 20) | (uint32_t)(0xfffff - i); }
FI float place_logit(uint64_t p) { return unordered((uint32_t)(p >> 20)); }
FI int place_token(uint64_t p) { return 0xfffff - (int)(p & 0xfffff); }

struct Row {
  float top;             // the largest logit
  float by_bin, by_bin_low;  // 128 / T as the sum of two
  double by_t;           // 1 / T
  FI void set(float top_, float t) {
    top = top_;
    by_t = 1.0 / (double)t;
    // (under T = 2^-90, where anything below the top lies below the bins, as for that)
    const double f = fmin(128.0 * by_t, 0x1p97);
    by_bin = (float)f;
    by_bin_low = (float)(f - (double)by_bin);
  }
  FI double weight(float x) const { return x == top ? 1.0 : exp(-(((double)top - (double)x) * by_t)); }
  // The place among the bins, rounded: its whole part is the bin, kBins and more lie below them.
  // (It falls with x whatever is rounded.)
  FI float bin(float x) const { return x == top ? 0.0f : (top - x) * by_bin; }
  // What is missing from 1 of exp(-f / 128), f the place in the bin, to 2^-30: a's own rounding
  // and that of the difference are taken in.
  FI float shortfall(float x, float a) const {
    const float d = x == top ? 0.0f : top - x, y = d - top;
    float low = fmaf(d, by_bin, -a) + d * by_bin_low;
    if (x != top) low = fmaf((top - (d - y)) + (-x - y), by_bin, low);
    const float f = ((a - floorf(a)) + low) * 0.0078125f;
    return f * (1.0f - f * (0.5f - f * 0.16666667f));
  }
};

// f(logit, token) for the row, by all threads of the workgroup.
template <class T>
FI float logit(const T* p, int i);
template <>
FI float logit<uint16_t>(const uint16_t* p, int i) {
  return __builtin_bit_cast(float, (uint32_t)p[i] << 16);
}
template <>
FI float logit<float>(const float* p, int i) {
  return p[i];
}
template <class T, class F>
FI void each(const T* x, int n, F f) {
  constexpr int E = 16 / sizeof(T), U = 4;
  const int tid = threadIdx.x;
  const int head = min(n, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  if (tid < head) f(logit(x, tid), tid);
  const u32x4* v = reinterpret_cast<const u32x4*>(x + head);
  const int nv = (n - head) / E;
  for (int c = tid; c < nv; c += U * kNT) {
    u32x4 r[U];
#pragma unroll
    for (int y = 0; y < U; ++y)
      if (c + y * kNT < nv) r[y] = v[c + y * kNT];
#pragma unroll
    for (int y = 0; y < U; ++y) {
      if (c + y * kNT >= nv) break;
      const int i = head + (c + y * kNT) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t w = sizeof(T) == 4 ? r[y][e & 3] : r[y][e / 2];
        f(__builtin_bit_cast(float, sizeof(T) == 4 ? w : e & 1 ? w & 0xffff0000u : w << 16), i + e);
      }
    }
  }
  const int tail = head + nv * E + tid;
  if (tail < n) f(logit(x, tail), tail);
}

// f(logit, token) for the tokens of those threads of `each` whose numbers stand in a list.
template <class T, class F>
FI void again(const T* x, int n, const int* group, int groups, F f) {
  constexpr int E = 16 / sizeof(T);
  const int tid = threadIdx.x;
  const int head = min(n, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  if (tid < head) f(logit(x, tid), tid);
  const u32x4* v = reinterpret_cast<const u32x4*>(x + head);
  const int nv = (n - head) / E, per = (nv + kNT - 1) / kNT;
  for (int item = tid; item < groups * per; item += kNT) {
    const int g = item / per, c = group[g] + (item - g * per) * kNT;
    if (c >= nv) continue;
    const u32x4 r = v[c];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t w = sizeof(T) == 4 ? r[e & 3] : r[e / 2];
      f(__builtin_bit_cast(float, sizeof(T) == 4 ? w : e & 1 ? w & 0xffff0000u : w << 16), head + c * E + e);
    }
  }
  const int tail = head + nv * E + tid;
  if (tail < n) f(logit(x, tail), tail);
}

// Sums over the workgroup in a fixed order; every thread gets the result.
FI double wave_scan(double x, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
FI int wave_scan(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

struct Shared {
  union {
    unsigned long long hist[kBins];
    struct {
      unsigned long long list[kList];
      double upto[kList];  // sums of w up to and with the list's token
    };
  };
  double mass[kBins];      // sums of w up to and with the bin
  int count[kBins];        // tokens up to and with the bin
  int offset[kBins];       // of the bin's tokens in the list, or -1
  union {
    int cursor[kBins];
    int group[kNT];        // threads whose tokens are looked at again
  };
  double part[kNT / 64];
  int ipart[kNT / 64];
  float fpart[kNT / 64];
  int at, groups;
};

// A whole workgroup's scan; the total in `total`.
FI double scan(Shared& s, double x, double& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double in = wave_scan(x, lane);
  __syncthreads();
  if (lane == 63) s.part[wave] = in;
  __syncthreads();
  double before = 0.0;
  total = 0.0;
  for (int y = 0; y < kNT / 64; ++y) {
    if (y == wave) before = total;
    total += s.part[y];
  }
  return before + in;
}
FI int scan(Shared& s, int x, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int in = wave_scan(x, lane);
  __syncthreads();
  if (lane == 63) s.ipart[wave] = in;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int y = 0; y < kNT / 64; ++y) {
    if (y == wave) before = total;
    total += s.ipart[y];
  }
  return before + in;
}

// Where the list is too short for the tokens of the bins that matter (many equal or nearly
// equal logits): the last place `to` in a bin for which the tokens of the bin up to it are at
// most / sum to what is asked for, found bit by bit with a walk over the row for each.
// count > 0: the count-th token of the bin.  Otherwise the first token at which `base` and the
// sum of w reach `target` (strict: pass it); the last of the bin where none does.
template <class T>
FI uint64_t search(Shared& s, const T* x, int n, const Row& row, int bin, int count, double base, double target,
                   bool strict, int& tokens, double& mass) {
  uint64_t to = 0;
  for (int bit = 51; bit >= -1; --bit) {  // (the last walk is for the result)
    const uint64_t cand = bit < 0 ? to : to | 1ull << bit;
    int c = 0;
    double m = 0.0;
    each(x, n, [&](float v, int i) {
      if ((int)fminf(row.bin(v), kBins) == bin && place(v, i) >= cand) {
        ++c;
        m += row.weight(v);
      }
    });
    double m_all;
    int c_all;
    scan(s, m, m_all);
    scan(s, c, c_all);
    const double sum = base + m_all;
    if (bit >= 0 && (count > 0 ? c_all >= count : c_all > 0 && (strict ? sum > target : sum >= target))) to = cand;
    tokens = c_all;
    mass = sum;
  }
  if (to == 0) {  // (sums from the bins may lie above those of the tokens by 2^-29: the last one)
    uint64_t last = ~0ull;
    each(x, n, [&](float v, int i) {
      if ((int)fminf(row.bin(v), kBins) == bin) last = min(last, place(v, i));
    });
#pragma unroll
    for (int d = 1; d < 64; d *= 2) last = min(last, (uint64_t)__shfl_xor((unsigned long long)last, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.list[threadIdx.x >> 6] = last;
    __syncthreads();
    for (int y = 0; y < kNT / 64; ++y) last = min(last, (uint64_t)s.list[y]);
    to = last;
  }
  return to;
}

template <class T>
__global__ __launch_bounds__(kNT) void sample_kernel(const SampleArgs a) {
  __shared__ Shared s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.x, n = a.vocab;
  const T* x = static_cast<const T*>(a.x) + r * a.stride;
  const float temperature = a.temperature ? a.temperature[r] : 1.0f;
  const int k_in = a.top_k ? a.top_k[r] : 0;
  const float p_in = a.top_p ? a.top_p[r] : 1.0f;
  const float m_in = a.min_p ? a.min_p[r] : 0.0f;
  const float u_in = a.u[r];
  auto answer = [&](int token, float logprob) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = logprob;
  };

  // the largest logit (NaN if there is one), and of each thread's
  float mine_top = -INFINITY;
  each(x, n, [&](float v, int) { mine_top = __builtin_elementwise_maximum(mine_top, v); });
  float top = mine_top;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = __builtin_elementwise_maximum(top, __shfl_xor(top, d));
  if (lane == 0) s.fpart[wave] = top;
  __syncthreads();
#pragma unroll
  for (int y = 0; y < kNT / 64; ++y) top = __builtin_elementwise_maximum(top, s.fpart[y]);
  if (!(top > -INFINITY) || !(temperature < INFINITY)) {
    if (tid == 0) answer(-1, NAN);
    return;
  }
  // The threads with a logit of at least a bound, whose tokens are all that has to be looked
  // at for those of at least that.
  auto list_groups = [&](float least) {
    if (tid == 0) s.groups = 0;
    __syncthreads();
    if (mine_top >= least) s.group[atomicAdd(&s.groups, 1)] = tid;
    __syncthreads();
  };
  if (temperature <= 0.0f) {  // the first of the largest
    list_groups(top);
    int first = n;
    again(x, n, s.group, s.groups, [&](float v, int i) {
      if (v == top) first = min(first, i);
    });
#pragma unroll
    for (int d = 1; d < 64; d *= 2) first = min(first, __shfl_xor(first, d));
    if (lane == 0) s.ipart[wave] = first;
    __syncthreads();
#pragma unroll
    for (int y = 0; y < kNT / 64; ++y) first = min(first, s.ipart[y]);
    if (tid == 0) answer(first, 0.0f);
    return;
  }
  Row row;
  row.set(top, temperature);
  const int k = k_in <= 0 || k_in > n ? n : k_in;
  const bool by_p = p_in < 1.0f, by_m = m_in > 0.0f;
  const double p = by_p ? fmax((double)p_in, 0.0) : 1.0;
  const double m = by_m ? fmin((double)m_in, 1.0) : 0.0;
  const double u = fmin(fmax(u_in == u_in ? (double)u_in : 0.0, 0.0), 1.0 - 0x1p-24);

  // The list in falling order, and the sums of w up to each of its tokens.
  auto sort_list = [&](int count) {
    int padded = 64;
    while (padded < count) padded *= 2;
    for (int i = count + tid; i < padded; i += kNT) s.list[i] = 0;  // (below every token)
    __syncthreads();
    for (int size = 2; size <= padded; size *= 2)  // bitonic
      for (int step = size / 2; step > 0; step /= 2) {
        for (int i = tid; i < padded / 2; i += kNT) {
          const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
          const unsigned long long p0 = s.list[lo], p1 = s.list[hi];
          if ((p0 < p1) == ((lo & size) == 0)) {
            s.list[lo] = p1;
            s.list[hi] = p0;
          }
        }
        // (up to 128 numbers are one wave's)
        if (padded > 128) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
      }
    if (padded <= 128) __syncthreads();
    constexpr int PT = kList / kNT;  // a thread has consecutive ones
    const int per = count <= kNT ? 1 : PT;
    double w[PT], run = 0.0, all;
#pragma unroll
    for (int y = 0; y < PT; ++y) {
      const int i = per * tid + y;
      w[y] = y < per && i < count ? row.weight(place_logit(s.list[i])) : 0.0;
      run += w[y];
    }
    run = scan(s, run, all) - run;
#pragma unroll
    for (int y = 0; y < PT; ++y) {
      run += w[y];
      if (y < per) s.upto[per * tid + y] = run;
    }
    __syncthreads();
  };
  // Items 0 .. c - 1 for which f holds, those a prefix of them.
  auto prefix = [&](int c, auto f) {
    if (c <= kNT) return __syncthreads_count(tid < c && f(tid));
    int got = 0;
    for (int i = tid; i < c; i += kNT) got += f(i);
    int all;
    scan(s, got, all);
    return all;
  };

  // Where the tokens that stay are few and a bound tells which can be among them, those are
  // listed and the rest is not looked at again: of k tokens none lies below the k-th largest of
  // the threads' maxima; min_p alone bounds the logit itself.
  const bool by_k = k <= kFew;
  if (by_k || (by_m && !by_p && k == n)) {
    float least;
    if (by_k) {
      const uint32_t key = ordered(mine_top);  // (the upper 16 bits are bound enough)
      uint32_t to = 0;
      for (int bit = 31; bit >= 16; --bit)
        if (__syncthreads_count(key >= (to | 1u << bit)) >= k) to |= 1u << bit;
      least = unordered(to);
      if (!(least >= -FLT_MAX)) least = -FLT_MAX;  // (also the words of a NaN; -infinity never stays)
    } else {
      least = (float)((double)top + log(m) * temperature * (1.0 + 1e-6) - fabs((double)top) * 0x1p-22);
      if (!(least <= top)) least = top;  // (+infinity)
    }
    if (tid == 0) s.at = 0;
    list_groups(least);
    again(x, n, s.group, s.groups, [&](float v, int i) {
      if (v >= least) {
        const int at = atomicAdd(&s.at, 1);
        if (at < kList) s.list[at] = place(v, i);
      }
    });
    __syncthreads();
    const int count = s.at;
    __syncthreads();
    if (count <= kList) {
      sort_list(count);
      int best = min(k, count);
      if (by_p) {
        const double target = p * s.upto[best - 1];
        best = min(best, prefix(best, [&](int i) { return s.upto[i] < target; }) + 1);
      }
      if (by_m) best = max(prefix(best, [&](int i) { return row.weight(place_logit(s.list[i])) >= m; }), 1);
      const double total = s.upto[best - 1], target = u * total;
      const int at = min(prefix(best, [&](int i) { return s.upto[i] <= target; }), best - 1);
      if (tid == 0) {
        const uint64_t drawn = s.list[at];
        answer(place_token(drawn), (float)log(row.weight(place_logit(drawn)) / total));
      }
      return;
    }
  }

  // counts and shortfalls of the bins; a thread has kBPT bins after each other
#pragma unroll
  for (int y = 0; y < kBPT; ++y) s.hist[tid + y * kNT] = 0;
  __syncthreads();
  each(x, n, [&](float v, int) {
    const float place = row.bin(v);
    if (place < kBins)
      atomicAdd(&s.hist[(int)place], (1ull << kFracBits) +
                                         (unsigned long long)(uint32_t)rintf(row.shortfall(v, place) * 0x1p30f));
  });
  __syncthreads();
  int mine[kBPT], in_bins = 0;
  double sum = 0.0;
  {
    double m_mine[kBPT], edge = exp(-0x1p-7 * (kBPT * tid));
    int c_all = 0;
    double m_all = 0.0;
#pragma unroll
    for (int y = 0; y < kBPT; ++y) {
      const unsigned long long raw = s.hist[kBPT * tid + y];
      mine[y] = (int)(raw >> kFracBits);
      m_mine[y] = ((double)mine[y] - (double)(raw & ((1ull << kFracBits) - 1)) * 0x1p-30) * edge;
      edge *= 0.992217938260243;  // exp(-1/128)
      c_all += mine[y];
      m_all += m_mine[y];
    }
    double m_up = scan(s, m_all, sum) - m_all;
    int c_up = scan(s, c_all, in_bins) - c_all;
#pragma unroll
    for (int y = 0; y < kBPT; ++y) {
      s.mass[kBPT * tid + y] = m_up += m_mine[y];
      s.count[kBPT * tid + y] = c_up += mine[y];
    }
  }
  __syncthreads();
  sum = s.mass[kBins - 1];  // (as the bins have it)
  auto mass_before = [&](int b) { return b > 0 ? s.mass[b - 1] : 0.0; };
  auto count_before = [&](int b) { return b > 0 ? s.count[b - 1] : 0; };
  // The number of bins for which f holds, those a prefix of them.
  auto bins_with = [&](auto f) {
    const int t = __syncthreads_count(f(kBPT * tid + kBPT - 1));
    int b = kBPT * t;
    if (t < kNT)
#pragma unroll
      for (int y = 0; y < kBPT - 1; ++y) b += f(kBPT * t + y);
    return b;
  };
  // the bin in which the sum reaches (strict: passes) a target
  auto bin_of = [&](double target, bool strict) {
    return min(bins_with([&](int b) { return strict ? s.mass[b] <= target : s.mass[b] < target; }), kBins - 1);
  };

  // The bins in which the borders can lie.
  const int bk = bins_with([&](int b) { return s.count[b] < k; });  // kBins: below them
  const double sk_lo = bk < kBins ? mass_before(bk) : sum, sk_hi = bk < kBins ? s.mass[bk] : sum;
  const int bp_lo = by_p ? bin_of(p * sk_lo, false) : kBins, bp_hi = by_p ? bin_of(p * sk_hi, false) : kBins;
  const double am = by_m ? -128.0 * log(m) : kBins;
  const int bm = am < kBins ? (int)am : kBins;
  const int be_lo = min(min(bk, bm), bp_lo), be_hi = min(min(bk, bm), bp_hi);
  const double total_lo = be_lo < kBins ? fmax(mass_before(be_lo), 1.0) : sum;
  const double total_hi = be_hi < kBins ? s.mass[be_hi] : sum;
  const int bd_lo = bin_of(u * total_lo, true), bd_hi = min(bin_of(u * total_hi, true), be_hi);
  int in_list, here = 0;
  bool wanted[kBPT];
#pragma unroll
  for (int y = 0; y < kBPT; ++y) {
    const int b = kBPT * tid + y;
    wanted[y] = b == bk || (by_p && b >= bp_lo && b <= bp_hi) || b == bm || (b >= bd_lo && b <= bd_hi);
    here += wanted[y] ? mine[y] : 0;
  }
  int off = scan(s, here, in_list) - here;

  int best = n;          // tokens that stay, and their sum
  double total = sum;
  uint64_t drawn;
  if (in_list <= kList) {
#pragma unroll
    for (int y = 0; y < kBPT; ++y) {
      s.offset[kBPT * tid + y] = wanted[y] ? off : -1;
      s.cursor[kBPT * tid + y] = 0;
      off += wanted[y] ? mine[y] : 0;
    }
    const float past = min(max(max(bk < kBins ? bk : 0, bm < kBins ? bm : 0), max(by_p ? bp_hi : 0, bd_hi)), kBins - 1) + 1;
    __syncthreads();
    each(x, n, [&](float v, int i) {
      const float at = row.bin(v);
      if (at < past) {
        const int b = (int)at;
        if (s.offset[b] >= 0) s.list[s.offset[b] + atomicAdd(&s.cursor[b], 1)] = place(v, i);
      }
    });
    __syncthreads();
    sort_list(in_list);
    // sum up to and with the c-th token of a bin (c = 0: before it)
    auto sum_at = [&](int b, int c) {
      const int o = s.offset[b];
      return mass_before(b) + (c > 0 ? s.upto[o + c - 1] - (o > 0 ? s.upto[o - 1] : 0.0) : 0.0);
    };
    auto tokens_of = [&](int b) { return s.count[b] - count_before(b); };
    if (bk < kBins) {
      best = k;
      total = sum_at(bk, k - count_before(bk));
    }
    if (by_p) {
      const double target = p * total;
      const int b = min(max(bin_of(target, false), bp_lo), bp_hi);
      const int c = min(prefix(tokens_of(b), [&](int i) { return sum_at(b, i + 1) < target; }) + 1, tokens_of(b));
      const int stay = max(count_before(b) + c, 1);
      if (stay < best) {
        best = stay;
        total = sum_at(b, c);
      }
    }
    if (bm < kBins) {
      const int c = prefix(tokens_of(bm), [&](int i) { return row.weight(place_logit(s.list[s.offset[bm] + i])) >= m; });
      const int stay = max(count_before(bm) + c, 1);
      if (stay < best) {
        best = stay;
        total = sum_at(bm, c);
      }
    }
    total = fmax(total, 1.0);
    const double target = u * total;
    const int b = min(max(bin_of(target, true), bd_lo), bd_hi);
    const int c = min(prefix(tokens_of(b), [&](int i) { return sum_at(b, i + 1) <= target; }), tokens_of(b) - 1);
    // (a sum that rounds past the last one that stays: that one, in the same bin)
    drawn = s.list[s.offset[b] + min(c, max(best - count_before(b), 1) - 1)];
  } else {
    int tokens;
    double mass;
    if (bk < kBins) {
      best = k;
      search(s, x, n, row, bk, k - count_before(bk), mass_before(bk), 0.0, false, tokens, mass);
      total = mass;
    }
    if (by_p) {
      const double target = p * total;
      const int b = bin_of(target, false);
      search(s, x, n, row, b, 0, mass_before(b), target, false, tokens, mass);
      const int stay = max(count_before(b) + tokens, 1);
      if (stay < best) {
        best = stay;
        total = mass;
      }
    }
    if (bm < kBins) {
      int c = 0;
      double w = 0.0;
      each(x, n, [&](float v, int) {
        if ((int)fminf(row.bin(v), kBins) == bm && row.weight(v) >= m) {
          ++c;
          w += row.weight(v);
        }
      });
      double w_all;
      int c_all;
      scan(s, w, w_all);
      scan(s, c, c_all);
      const int stay = max(count_before(bm) + c_all, 1);
      if (stay < best) {
        best = stay;
        total = mass_before(bm) + w_all;
      }
    }
    total = fmax(total, 1.0);
    const double target = u * total;
    const int b = min(bin_of(target, true), be_hi);
    drawn = search(s, x, n, row, b, 0, mass_before(b), target, true, tokens, mass);
    if (count_before(b) + tokens > best)
      drawn = search(s, x, n, row, b, max(best - count_before(b), 1), mass_before(b), 0.0, false, tokens, mass);
  }
  if (tid == 0) answer(place_token(drawn), (float)log(row.weight(place_logit(drawn)) / total));
}

}  // namespace

size_t sample_workspace_bytes(int dtype, int n, int vocab) { return 0; }

hipError_t launch_sample(int dtype, const SampleArgs& a, hipStream_t s) {
  if (dtype == HF_BF16)
    sample_kernel<uint16_t><<<(unsigned)a.n, kNT, 0, s>>>(a);
  else
    sample_kernel<float><<<(unsigned)a.n, kNT, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace hf
