// The next token from a row of logits and a given random number (Table 1's
// AI_TRANSFORM): temperature, top-k, top-p, min-p, inverse distribution in the
// order of ids.
//
// A workgroup of 16 or 4 waves per row, each wave a run of ids; every pass reads the row again,
// from the L2 where that still holds it.  (Held in registers, 32 logits per thread, a row per CU, the reading of 4,096 rows
// of 32,000 did not overlap the arithmetic: 580 us against 465.  With no more rows than CUs, where there is nothing
// to overlap, it has not been measured.)
//
// Bound: the vector unit, fp64 first of all (a weight is about 20 fp64 instructions), on the CUs that
// have a row; one row after its latencies, a pass per 2 us or so.  Rows of 32,000 fp32 logits in launches one after
// another, us:
//             temperature 0  no filter  min-p 0.05  top-k 50  top-k 1,000  top-k 2,000  top-p 0.9
//   1 row            8          16         22          20         28          45           41
//   256 rows         9          20         28          22         30          52           47
//   2,048 rows      42         135        164          88        225         244          280
//   the same cold   53         134        168         100        239         257          289
// The rows of the first three lines (262 MB in the third) are those of the launch before, so what the 256 MB of
// last-level cache keep of them is not read from HBM; "cold" are four such matrices in turn (55 us a reading).
// 96 rows of 131,071 bf16 logits with top-k 1,000 and top-p 0.95 take 60, on 96 of the 256 CUs.
// The 16-wave kernels with filters are at their 128 registers (16 waves on a CU) and spill 3 to 5 more to scratch (16 to 24
// bytes per lane), as the 4-wave ones of fp32 do by 1 or 2.
//
// Weights are whole numbers, round(2^S exp((x - m) / T)) from fp64 exponentials
// (below), S such that a whole vocabulary's sum fits 62 bits: sums do not
// depend on their order, so they may come from LDS atomics, and a weight keeps
// 2^-47 of the largest at 32,000 tokens.  (In 32 bits a border between two tokens
// moves by 1e-7 of the sum, which is a share of 3e-3 of all random numbers with
// 32,000 borders.  Here it moves by less than V^2 2^-61: V roundings of half a step, in the sum up to it and in the whole,
// which is 2^S >= 2^61 / V at least.)
//
// All filters keep a prefix of the tokens in descending order, equal ones by
// ascending id, so the kept set is a threshold (x, id).  Top-k and top-p find theirs
// the same way, by counts or by weights: a histogram over the distance to the
// maximum (2,048 bins in LDS), the bin in which the count or the sum reaches its
// target, and in that bin the token itself, by comparing its tokens (60 or so) with each other.
// Where top-k leaves few tokens (draw_few) the steps after it are taken among those alone.
// A bin with more than CAP tokens (equal logits, a far outlier) is halved bit by bit instead, 57 further passes over the
// row: logits of four levels only, 32,000 of them, take 372 us with top-k and 696 with top-p where a row of the table
// takes 20 and 41 (1,024 rows 1.5 and 2.9 ms), and 16-bit logits around 8 with 131,072 tokens, whose steps of 1/32 or 1/16
// hold more than CAP tokens, 195 with top-p 0.9 (700 rows 738).
#include "aiq_internal.h"
#include "dev_util.h"

#include <type_traits>

namespace aiq {

constexpr int SW_MAX = 16;            // waves
constexpr int BINS = 2048;
// tokens that a workgroup of SW waves gathers and compares with each other (LDS for four small ones on a CU)
constexpr int cap(int sw) { return sw == 16 ? 2048 : 1024; }

template <int DT>
struct Logits4 {   // 4 logits, aligned to one
  typedef float T;
  T v[4];
} __attribute__((packed, aligned(4)));
template <>
struct Logits4<AIQ_F16> {
  typedef uint16_t T;
  T v[4];
} __attribute__((packed, aligned(2)));
template <>
struct Logits4<AIQ_BF16> {
  typedef uint16_t T;
  T v[4];
} __attribute__((packed, aligned(2)));

template <int DT>
__device__ __forceinline__ float to_logit(typename Logits4<DT>::T v) {   // NaN: never taken
  float x;
  if constexpr (DT == AIQ_F32)
    x = v;
  else
    x = DT == AIQ_F16 ? h2f(v) : bf2f(v);
  return fmaxf(x, -INFINITY);
}

// Bit pattern that orders as the values do (-0 as 0)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr double ROUND = 0x1.8p52;   // x + ROUND: x rounded to a whole number, in the low bits
struct Weigh {
  double c;         // log2(e) / T
  double d0;        // a distance whose weight rounds to 0
  double least;     // min_p * 2^S
  int s;            // S
  float m;
  // 2^S exp((x - m) / T), not rounded yet: 2^y = 2^n 2^f with n the nearest whole
  // number and 2^f on [-1/2, 1/2] as 1 + f Q(f), Q of degree 8 through the
  // Chebyshev nodes (relative error 4e-14); exactly 2^S at the maximum.
  __device__ __forceinline__ double real(float x) const {
    const double d = fmax(static_cast<double>(x) - static_cast<double>(m), d0);
    const double t = fma(d, c, ROUND), f = fma(d, c, ROUND - t);
    double q = 0x1.b638809761cfdp-24;
    q = fma(q, f, 0x1.63d13636b876dp-20);
    q = fma(q, f, 0x1.ffcb9515b4237p-17);
    q = fma(q, f, 0x1.4308ac85aa3bbp-13);
    q = fma(q, f, 0x1.5d87fe86fe84cp-10);
    q = fma(q, f, 0x1.3b2ab7181b759p-7);
    q = fma(q, f, 0x1.c6b08d7047e52p-5);
    q = fma(q, f, 0x1.ebfbdff823cedp-3);
    q = fma(q, f, 0x1.62e42fefa39efp-1);
    const int64_t z = __double_as_longlong(fma(q, f, 1.0));   // times 2^(n + S), in the exponent's bits
    const uint32_t n = static_cast<uint32_t>(__double_as_longlong(t)) + s;
    return __longlong_as_double(z + (static_cast<int64_t>(n << 20) << 32));
  }
  // the nearest whole number of a value below 2^51, with BIAS added
  static __device__ __forceinline__ uint64_t biased(double v) {
    return static_cast<uint64_t>(__double_as_longlong(v + 0x1p52));
  }
  static constexpr uint64_t BIAS = 0x433ull << 52;
  __device__ __forceinline__ uint64_t of(float x) const { return biased(real(x)) - BIAS; }
  __device__ __forceinline__ uint64_t kept(float x) const {   // 0 below min_p
    const double v = real(x);
    return v >= least ? biased(v) - BIAS : 0;
  }
};

__device__ __forceinline__ uint64_t shfl_u64(uint64_t v, int mask) {
  const uint32_t lo = __shfl_xor(static_cast<uint32_t>(v), mask), hi = __shfl_xor(static_cast<uint32_t>(v >> 32), mask);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
// v shifted or broadcast between lanes (0 where nothing comes), added
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_add_u64(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(v)), CTRL, ROWS, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(v >> 32)), CTRL, ROWS, 0xF, true);
  return v + ((static_cast<uint64_t>(hi) << 32) | lo);
}
// inclusive sum over the lanes up to this one: inside rows of 16 (row_shr 1, 2, 4, 8), then the last
// lane of a row to the next row, of a half to the other (row_bcast 15, 31)
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v) {
  v = dpp_add_u64<0x111, 0xF>(v);
  v = dpp_add_u64<0x112, 0xF>(v);
  v = dpp_add_u64<0x114, 0xF>(v);
  v = dpp_add_u64<0x118, 0xF>(v);
  v = dpp_add_u64<0x142, 0xA>(v);
  return dpp_add_u64<0x143, 0xC>(v);
}
__device__ __forceinline__ uint64_t last_lane(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(v)), 63);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(v >> 32)), 63);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) { return last_lane(wave_scan_u64(v)); }

struct SampleSums {
  uint64_t wave[SW_MAX];
  float lo[SW_MAX];
};
template <int SW>
struct SampleLds : SampleSums {
  static constexpr int CAP = cap(SW);
  uint64_t bin[BINS];
  uint64_t key[CAP];     // gathered tokens: (ordered bits of the logit, ~id)
  uint64_t w[CAP];
  uint64_t before, target;
  int32_t at, n;         // the bin, its tokens
  uint64_t last;         // the threshold, as a key
};

template <int SW>
__device__ __forceinline__ uint64_t block_sum(uint64_t v, SampleSums& s) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t t = 0;
#pragma unroll
  for (int w = 0; w < SW; ++w) t += s.wave[w];
  return t;
}

// A workgroup's row: f(logit, id) for every one of this thread's tokens, in
// ascending order of ids (-infinity past the end); all lanes call f together.
template <int DT, int AHEAD>   // AHEAD: rounds of logits in flight
struct Row {
  const typename Logits4<DT>::T* p;
  int V, rounds, id0;   // this thread's tokens: id0 + 256 * round + 0 .. 3
  bool inf;             // the maximum is +infinity: its tokens read as 0, the others as -infinity
  typedef typename Logits4<DT>::T T;
  typedef T Raw __attribute__((ext_vector_type(4)));
  static constexpr T NONE = DT == AIQ_F32 ? static_cast<T>(-INFINITY) : DT == AIQ_F16 ? static_cast<T>(0xFC00) : static_cast<T>(0xFF80);
  __device__ __forceinline__ Raw fetch(int it) const {
    const int id = id0 + it * 256;
    Raw y = {NONE, NONE, NONE, NONE};
    if (__builtin_amdgcn_readfirstlane(id) + 256 <= V) {   // all of the wave's
      const Logits4<DT> z = *reinterpret_cast<const Logits4<DT>*>(p + id);
      y = Raw{z.v[0], z.v[1], z.v[2], z.v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (id + e < V) y[e] = p[id + e];
    }
    return y;
  }
  __device__ __forceinline__ void values(const Raw& y, float (&v)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_logit<DT>(y[e]);
    if (inf) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] == INFINITY ? 0.f : -INFINITY;
    }
  }
  struct Ids {
    int first;
    __device__ __forceinline__ int operator[](int e) const { return first + e; }
  };
  static constexpr bool FEW = false;
  template <typename F>
  __device__ __forceinline__ void each4(F f) const {   // f(4 logits, their ids)
    Raw y[AHEAD];   // the next rounds, in flight
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
      if (d < rounds) y[d] = fetch(d);
#pragma unroll 1
    for (int it = 0; it < rounds; ++it) {
      float v[4];
      values(y[0], v);
#pragma unroll
      for (int d = 0; d + 1 < AHEAD; ++d) y[d] = y[d + 1];
      if (it + AHEAD < rounds) y[AHEAD - 1] = fetch(it + AHEAD);
      f(v, Ids{id0 + it * 256});
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    each4([&](const float (&v)[4], const Ids& id) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f(v[e], id[e]);
    });
  }
};

// Tokens gathered from a row, up to 4 per thread (an empty place: -infinity, behind every threshold).
struct List {
  static constexpr bool FEW = true;   // no more than CAP
  float x[4];
  int id[4];
  template <typename F>
  __device__ __forceinline__ void each4(F f) const {
    f(x, id);
  }
};

// tokens up to the threshold (xt, idt), the tokens kept so far
__device__ __forceinline__ bool upto(float x, int id, float xt, int idt) {
  return x > xt || (x == xt && id <= idt);
}
__device__ __forceinline__ uint64_t token_key(float x, int id) {   // larger is earlier
  return (static_cast<uint64_t>(order_key(x)) << 32) | static_cast<uint32_t>(~id);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t k = static_cast<uint32_t>(key >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ int key_id(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

// Bins of the distance to the maximum: `span` over all but the last, which takes what is beyond
struct Bins {
  float m, per;
  __device__ __forceinline__ Bins(float m_, float span) : m(m_), per(span > 0.f ? static_cast<float>(BINS - 1) / span : 0.f) {}
  __device__ __forceinline__ float place(float x) const { return fminf((m - x) * per, static_cast<float>(BINS - 1)); }
};

// The bin in which the counts or weights in `bin` (of all threads) reach the target that goal(total)
// gives: s.at, with s.before ahead of it.  Ends with a barrier.
template <int SW, typename T, typename G>
__device__ __forceinline__ void cross(const T* bin, G goal, SampleLds<SW>& s) {
  constexpr int PB = BINS / (64 * SW);
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  uint64_t mine = 0;
  for (int q = 0; q < PB; ++q) mine += bin[PB * tid + q];
  const uint64_t incl = wave_scan_u64(mine);
  if (lane == 63) s.wave[wv] = incl;
  __syncthreads();
  uint64_t before = incl - mine, total = 0;
#pragma unroll
  for (int x = 0; x < SW; ++x) {
    if (x < wv) before += s.wave[x];
    total += s.wave[x];
  }
  const uint64_t target = goal(total);
  if (before < target && target <= before + mine) {
    int q = 0;
    for (; q < PB - 1 && before + bin[PB * tid + q] < target; ++q) before += bin[PB * tid + q];
    s.at = PB * tid + q;
    s.before = before;
    s.target = target;
  }
  __syncthreads();
}

// Gathers the tokens that pred picks: s.n of them, the first CAP as keys.  All lanes together.
template <int SW>
__device__ __forceinline__ void gather(bool in, float x, int id, SampleLds<SW>& s) {
  const uint64_t b = __ballot(in);
  if (!b) return;
  const int lead = __builtin_ctzll(b);
  int slot = 0;
  if ((threadIdx.x & 63) == lead) slot = atomicAdd(&s.n, __popcll(b));
  slot = __shfl(slot, lead) + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(b >> 32),
                                                       __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(b), 0));
  if (in && slot < s.CAP) s.key[slot] = token_key(x, id);
}

// p_of top_p of a sum of weights, as a whole number in 1 .. total
__device__ __forceinline__ uint64_t share_of(double p, uint64_t total) {
  const double t = ceil(p * static_cast<double>(total));
  const uint64_t g = t < static_cast<double>(total) ? static_cast<uint64_t>(t) : total;
  return g ? g : 1;
}

// Moves the threshold (xt, idt) to the token at which the count (MASS: the sum of weights) of the
// tokens reaches its target: top_k, or top_p of the sum of the tokens kept so far.
template <int SW, bool MASS, typename R>
__device__ __forceinline__ void find(const R& row, const Weigh& w, double top, float span, float& xt, int& idt, SampleLds<SW>& s) {
  constexpr int SN = 64 * SW, CAP = cap(SW);
  const int tid = threadIdx.x, lane = tid & 63;
  typedef std::conditional_t<MASS, uint64_t, uint32_t> T;
  T* bin = reinterpret_cast<T*>(s.bin);
  const Bins bins(w.m, span);
  for (int b = tid; b < BINS; b += SN) bin[b] = 0;
  if (tid == 0) s.n = 0;
  __syncthreads();
  T rest = 0;   // the last bin's
  row.each4([&](const float (&x)[4], const auto& id) {
    bool in[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) in[e] = upto(x[e], id[e], xt, idt);
    if (!__any(in[0] || in[1] || in[2] || in[3])) return;
    T v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (MASS)
        v[e] = w.of(x[e]);
      else
        v[e] = 1;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int b = static_cast<int>(bins.place(x[e]));
      if (in[e] && b == BINS - 1) rest += v[e];
      if (in[e] && b < BINS - 1) atomicAdd(reinterpret_cast<std::conditional_t<MASS, unsigned long long, uint32_t>*>(&bin[b]), v[e]);
    }
  });
  const uint64_t all = wave_sum_u64(rest);
  if (lane == 0 && all)
    atomicAdd(reinterpret_cast<std::conditional_t<MASS, unsigned long long, uint32_t>*>(&bin[BINS - 1]), static_cast<T>(all));
  __syncthreads();
  cross<SW>(bin, [&](uint64_t total) -> uint64_t {
    return MASS ? share_of(top, total) : top < static_cast<double>(total) ? static_cast<uint64_t>(top) : total;
  }, s);
  const int at = s.at;
  const uint64_t before = s.before, target = s.target;
  const float from = static_cast<float>(at), to = at == BINS - 1 ? INFINITY : static_cast<float>(at + 1);
  auto in_bin = [&](float x, int id) {
    const float f = bins.place(x);
    return f >= from && f < to && upto(x, id, xt, idt);
  };
  row.each4([&](const float (&x)[4], const auto& id) {
    bool in[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) in[e] = in_bin(x[e], id[e]);
    if (!__any(in[0] || in[1] || in[2] || in[3])) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) gather(in[e], x[e], id[e], s);
  });
  __syncthreads();
  const int n = s.n;
  if (R::FEW || n <= CAP) {
    for (int i = tid; MASS && i < n; i += SN) s.w[i] = w.of(key_logit(s.key[i]));
    __syncthreads();
    int each = 64;   // threads per token
    while (each > 1 && n * each > SN) each >>= 1;
    for (int i0 = 0; i0 < n; i0 += SN / each) {
      const int i = i0 + tid / each;
      const uint64_t key = i < n ? s.key[i] : 0;
      uint64_t ahead = 0;   // of the bin's tokens ahead of this one
      for (int j = tid % each; j < n; j += each)
        if (s.key[j] > key) ahead += MASS ? s.w[j] : 1;
      for (int o = each / 2; o > 0; o >>= 1) ahead += shfl_u64(ahead, o);
      ahead += before;
      if (i < n && tid % each == 0 && ahead < target && target <= ahead + (MASS ? s.w[i] : 1)) s.last = key;
    }
  } else if constexpr (!R::FEW) {
    // the largest key K such that the bin's tokens with keys from K on reach the target, bit by bit
    uint32_t K = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t k = K | (1u << bit);
      uint64_t v = 0;
      row.each([&](float x, int id) {
        if (in_bin(x, id) && order_key(x) >= k) v += MASS ? w.of(x) : 1;
      });
      if (before + block_sum<SW>(v, s) >= target) K = k;
    }
    uint64_t above = 0;
    row.each([&](float x, int id) {
      if (in_bin(x, id) && order_key(x) > K) above += MASS ? w.of(x) : 1;
    });
    above = before + block_sum<SW>(above, s);
    // of the tokens with that key the first `t` ids do not reach it, the largest such t
    int t = 0;
    for (int bit = 24; bit >= 0; --bit) {
      uint64_t v = 0;
      const int u = t | (1 << bit);
      row.each([&](float x, int id) {
        if (id < u && in_bin(x, id) && order_key(x) == K) v += MASS ? w.of(x) : 1;
      });
      if (above + block_sum<SW>(v, s) < target) t = u;
    }
    if (tid == 0) s.last = (static_cast<uint64_t>(K) << 32) | static_cast<uint32_t>(~t);
  }
  __syncthreads();
  xt = key_logit(s.last);
  idt = key_id(s.last);
  __syncthreads();
}

// The sum of weights, in the order of ids, that the drawn token is the first to exceed
__device__ __forceinline__ uint64_t draw_target(float u, uint64_t total) {
  if (!(u < 1.f)) return total - 1;
  const double t = static_cast<double>(u) * static_cast<double>(total);
  const uint64_t g = t > 0.0 ? static_cast<uint64_t>(t) : 0;
  return g < total ? g : total - 1;
}

// Top-k with what follows it among few tokens: of the 4 maxima that each thread has (of every fourth of its
// tokens), k lie in the bins up to one, and so at least k tokens do; where they are no more than CAP, the filters and the
// draw need these alone.  False: they are more (or fewer maxima than k).
template <int SW, typename R>
__device__ __forceinline__ bool draw_few(const R& row, const Weigh& w, const float (&most)[4], const SampleArgs& a,
                                         int64_t r, float u, SampleLds<SW>& s) {
  constexpr int SN = 64 * SW, CAP = cap(SW), PER = CAP / SN;   // gathered tokens per thread
  const int tid = threadIdx.x;
  uint32_t* bin = reinterpret_cast<uint32_t*>(s.bin);
  const Bins bins(w.m, 32.f);
  for (int b = tid; b < BINS; b += SN) bin[b] = 0;
  if (tid == 0) {
    s.n = 0;
    s.at = -1;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (most[q] > -INFINITY) atomicAdd(&bin[static_cast<int>(bins.place(most[q]))], 1u);
  __syncthreads();
  cross<SW>(bin, [&](uint64_t total) { return static_cast<uint64_t>(a.top_k); }, s);
  const int at = s.at;
  if (at < 0 || at == BINS - 1) return false;
  const float to = static_cast<float>(at + 1);
  row.each4([&](const float (&x)[4], const auto& id) {
    bool in[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) in[e] = (w.m - x[e]) * bins.per < to;
    if (!__any(in[0] || in[1] || in[2] || in[3])) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) gather(in[e], x[e], id[e], s);
  });
  __syncthreads();
  const int n = s.n;
  if (n > CAP) {
    __syncthreads();   // every wave has read the count that the next step clears
    return false;
  }
  const int k = a.top_k < n ? a.top_k : n;
  if (n <= 128) {   // by comparing all with all, SN / 128 threads or more per token: fewer barriers
    const int each = SN / (n <= 64 ? 64 : 128), i = tid / each;
    for (int j = tid; j < n; j += SN) s.w[j] = w.of(key_logit(s.key[j]));
    __syncthreads();
    const uint64_t key = i < n ? s.key[i] : 0, mine = i < n ? s.w[i] : 0;
    uint64_t ahead = 0;
    int rank = 0;
    for (int j = tid % each; j < n; j += each)
      if (s.key[j] > key) {
        ahead += s.w[j];
        ++rank;
      }
    for (int o = each / 2; o > 0; o >>= 1) {
      ahead += shfl_u64(ahead, o);
      rank += __shfl_xor(rank, o);
    }
    const bool lead = i < n && tid % each == 0;
    uint64_t total = block_sum<SW>(lead && rank < k ? mine : 0, s);
    const uint64_t target = a.top_p < 1.0 ? share_of(a.top_p, total) : total;
    const uint64_t keep = i < n && rank < k && ahead < target ? w.kept(key_logit(key)) : 0;
    if (lead) s.w[i] = keep;
    total = block_sum<SW>(lead ? keep : 0, s);
    const uint64_t goal = draw_target(u, total);
    uint64_t below = 0;   // kept weights of lower ids: larger low words
    for (int j = tid % each; j < n; j += each)
      if (static_cast<uint32_t>(s.key[j]) > static_cast<uint32_t>(key)) below += s.w[j];
    for (int o = each / 2; o > 0; o >>= 1) below += shfl_u64(below, o);
    if (lead && below <= goal && goal < below + keep) a.token[r] = key_id(key);
    __syncthreads();
    return true;
  }
  // the same steps as over a row, with the tokens in registers
  static_assert(PER >= 1 && PER <= 4);
  List list;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int i = tid + q * SN;
    const bool is = q < PER && i < n;
    const uint64_t key = is ? s.key[i] : 0;
    list.x[q] = is ? key_logit(key) : -INFINITY;
    list.id[q] = is ? key_id(key) : 0;
  }
  __syncthreads();
  float xt = -INFINITY;
  int idt = -1;
  const float span = to / bins.per;
  if (k < n) find<SW, false>(list, w, k, span, xt, idt, s);
  if (a.top_p < 1.0) find<SW, true>(list, w, a.top_p, span, xt, idt, s);
  // the draw: kept weights in bins of ids
  uint64_t* ids = reinterpret_cast<uint64_t*>(s.bin);
  const float per = static_cast<float>(BINS) / static_cast<float>(a.vocab);
  auto place = [&](int id) { return static_cast<int>(fminf(static_cast<float>(id) * per, static_cast<float>(BINS - 1))); };
  for (int b = tid; b < BINS; b += SN) ids[b] = 0;
  if (tid == 0) s.n = 0;
  __syncthreads();
  uint64_t keep[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    keep[q] = upto(list.x[q], list.id[q], xt, idt) ? w.kept(list.x[q]) : 0;
    if (keep[q]) atomicAdd(reinterpret_cast<unsigned long long*>(&ids[place(list.id[q])]), static_cast<unsigned long long>(keep[q]));
  }
  __syncthreads();
  cross<SW>(ids, [&](uint64_t total) { return draw_target(u, total) + 1; }, s);
  const uint64_t before = s.before, target = s.target;
#pragma unroll
  for (int q = 0; q < PER; ++q) gather(keep[q] != 0 && place(list.id[q]) == s.at, list.x[q], list.id[q], s);
  __syncthreads();
  const int m = s.n;
  for (int i = tid; i < m; i += SN) s.w[i] = w.of(key_logit(s.key[i]));
  __syncthreads();
  for (int i = tid; i < m; i += SN) {
    const uint32_t key = static_cast<uint32_t>(s.key[i]);
    uint64_t below = before;   // with the lower ids of the bin: larger low words
    for (int j = 0; j < m; ++j)
      if (static_cast<uint32_t>(s.key[j]) > key) below += s.w[j];
    if (below < target && target <= below + s.w[i]) a.token[r] = key_id(s.key[i]);
  }
  __syncthreads();
  return true;
}

template <int DT, int SW, bool FILTER>
__global__ __launch_bounds__(64 * SW, SW == SW_MAX || FILTER ? 4 : 8) void k_sample(SampleArgs a) {
  constexpr int SN = 64 * SW;
  __shared__ std::conditional_t<FILTER, SampleLds<SW>, SampleSums> s;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int V = a.vocab;
  int64_t rows = a.n_rows;
  if (a.n_ptr && *a.n_ptr < rows) rows = *a.n_ptr;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    Row<DT, SW == SW_MAX || FILTER ? 4 : 2> row;   // (64 registers a lane in the last)
    row.p = static_cast<const typename Logits4<DT>::T*>(a.logits) + r * a.ld;
    row.V = V;
    row.rounds = (V + SN * 4 - 1) / (SN * 4);
    const int run = row.rounds * 256;   // ids per wave
    row.id0 = wv * run + lane * 4;
    row.inf = false;
    // the maximum and the least finite logit; at temperature 0 the lowest id that has the maximum
    float best = -INFINITY, least = INFINITY;
    const bool greedy = a.temperature == 0.0;
    int first = INT32_MAX;
    float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};   // of every fourth of the thread's tokens
    if (greedy)
      row.each([&](float x, int id) {
        first = x > best ? id : first;
        best = fmaxf(best, x);
      });
    else {
      row.each4([&](const float (&v)[4], const auto& id) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          most[e] = fmaxf(most[e], v[e]);
          if (FILTER) least = v[e] > -INFINITY ? fminf(least, v[e]) : least;
        }
      });
      best = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    }
    uint64_t top = (static_cast<uint64_t>(order_key(best)) << 32) | static_cast<uint32_t>(~first);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t y = shfl_u64(top, o);
      top = y > top ? y : top;
      least = fminf(least, __shfl_xor(least, o));
    }
    __syncthreads();   // (the row before)
    if (lane == 0) {
      s.wave[wv] = top;
      s.lo[wv] = least;
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < SW; ++x) {
      top = s.wave[x] > top ? s.wave[x] : top;
      least = fminf(least, s.lo[x]);
    }
    __syncthreads();
    const uint32_t mk = static_cast<uint32_t>(top >> 32);
    Weigh w;
    w.m = __uint_as_float(mk & 0x80000000u ? mk & 0x7FFFFFFFu : ~mk);
    if (w.m == -INFINITY || greedy) {
      if (tid == 0) a.token[r] = w.m == -INFINITY ? 0 : static_cast<int>(~static_cast<uint32_t>(top));
      continue;
    }
    if (w.m == INFINITY) {
      row.inf = true;
      w.m = least = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) most[q] = most[q] == INFINITY ? 0.f : -INFINITY;
    }
    const int bits = 32 - __builtin_clz(static_cast<uint32_t>(V));
    // (temperatures past 1e200 are that: finite logits are at most 2^129 apart and weigh the same all the same, and the
    // distance d0 stays finite, so that -infinity weighs nothing)
    w.c = 1.4426950408889634 * fmax(fmin(1.0 / a.temperature, 1e300), 1e-200);
    w.s = bits > 12 ? 62 - bits : 50;
    w.d0 = -(w.s + 4.0) / w.c;
    w.least = a.min_p * static_cast<double>(1ull << w.s);
    float xt = -INFINITY;   // all but -infinity
    int idt = -1;
    const float range = w.m - least;
    const float u = a.u[a.u_row ? a.u_row[*a.u_base + a.u_add + r] * a.u_ld + a.u_at : r];
    if constexpr (FILTER) {
    if (a.top_k > 0 && draw_few<SW>(row, w, most, a, r, u, s)) continue;
    if (a.top_k > 0) find<SW, false>(row, w, a.top_k, fminf(range, 40.f), xt, idt, s);
    if (a.top_p < 1.0) {
      // tokens with less than (1 - top_p) / V of the maximum's weight are behind the last one kept
      const double far = a.temperature * log(V / (1.0 - a.top_p)) * 1.0001;
      find<SW, true>(row, w, a.top_p, fminf(range, static_cast<float>(far)), xt, idt, s);
    }
    }
    // the wave, then the round, then the token that the random number falls into
    uint64_t mine = 0;
    if (!FILTER) {
      row.each([&](float x, int id) { mine += Weigh::biased(w.real(x)); });
      mine -= static_cast<uint64_t>(row.rounds) * 4 * Weigh::BIAS;
    } else {
      row.each4([&](const float (&x)[4], const auto& id) {
        bool in[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) in[e] = upto(x[e], id[e], xt, idt);
        if (!__any(in[0] || in[1] || in[2] || in[3])) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint64_t v = w.kept(x[e]);
          mine += in[e] ? v : 0;
        }
      });
    }
    mine = wave_sum_u64(mine);
    if (lane == 0) s.wave[wv] = mine;
    __syncthreads();
    uint64_t total = 0, at = 0;
#pragma unroll
    for (int x = 0; x < SW; ++x) {
      if (x == wv) at = total;
      total += s.wave[x];
    }
    const uint64_t target = draw_target(u, total);   // at least the maximum is kept
    if (target >= at && target - at < mine) {   // this wave's
      for (int it = 0; it < row.rounds; ++it) {
        float v[4];
        row.values(row.fetch(it), v);
        uint64_t k[4], all = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int id = row.id0 + it * 256 + e;
          k[e] = FILTER ? upto(v[e], id, xt, idt) ? w.kept(v[e]) : 0 : w.of(v[e]);
          all += k[e];
        }
        const uint64_t incl = at + wave_scan_u64(all);
        at = last_lane(incl);
        if (at > target) {
          const uint64_t hit = __ballot(incl > target);
          if (lane == __builtin_ctzll(hit)) {
            uint64_t c = incl - all;
            int e = 0;
            for (; e < 3; ++e) {
              c += k[e];
              if (c > target) break;
            }
            a.token[r] = row.id0 + it * 256 + e;
          }
          break;
        }
      }
    }
  }
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(a.n_rows < 65536 ? a.n_rows : 65536));
  const bool filter = a.temperature > 0.0 && (a.top_k > 0 || a.top_p < 1.0 || a.min_p > 0.0);
  // 16 waves per row up to the rows that leave CUs without one of theirs, 4 beyond.  Rows of 32,000 logits, 16 waves
  // against 4: without filters 512 rows 39 us against 48, 700 rows 52 against 58, 1,023 rows 68 against 71; top-p 512 rows
  // 91 against 106, 640 rows 129 against 129, 1,023 rows 177 against 155; top-k 512 rows 41 against 36, 640 58 against 38.
  // Also where only 16 waves gather the top-k (draw_few's bound lets in up to twice as many): 2,048 rows with top-k 700
  // 218 us against 303, with 500 212 against 121.
  const bool wide = a.n_rows < (!filter ? 1024 : a.top_k > 0 ? 512 : 640) ||
                    (a.top_k > cap(4) / 2 && a.top_k <= cap(SW_MAX) / 2);
#define AIQ_SAMPLE_K(DT_, SW_, F_) hipLaunchKernelGGL((k_sample<DT_, SW_, F_>), grid, dim3(64 * SW_), 0, s, a)
#define AIQ_SAMPLE(DT_)                                        \
  if (wide && filter) AIQ_SAMPLE_K(DT_, SW_MAX, true);         \
  else if (wide) AIQ_SAMPLE_K(DT_, SW_MAX, false);             \
  else if (filter) AIQ_SAMPLE_K(DT_, 4, true);                 \
  else AIQ_SAMPLE_K(DT_, 4, false)
  if (a.dtype == AIQ_F32) {
    AIQ_SAMPLE(AIQ_F32);
  } else if (a.dtype == AIQ_F16) {
    AIQ_SAMPLE(AIQ_F16);
  } else if (a.dtype == AIQ_BF16) {
    AIQ_SAMPLE(AIQ_BF16);
  } else {
    return hipErrorInvalidValue;
  }
#undef AIQ_SAMPLE
#undef AIQ_SAMPLE_K
  return hipGetLastError();
}

}  // namespace aiq
