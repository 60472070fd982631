// The next token from a row of logits and a given random number (Table 1's
// AI_TRANSFORM): temperature, top-k, top-p, min-p, inverse distribution in the
// order of ids.
//
// A workgroup per row.  Weights are whole numbers, round(2^S exp((x - m) / T)) from fp64
// exponentials, S such that a whole vocabulary's sum fits 63 bits: sums do not depend on
// their order, so they may come from LDS atomics, and a weight keeps 2^-47 of the
// largest at 32,000 tokens.  All three filters keep a prefix of the tokens in
// descending order of logits, so the kept set is a threshold: the prefix's last
// value and, where only some of the tokens equal to it belong, the last id of
// those.  It is found digit by digit of the value's ordered bit pattern, counting
// tokens (top-k) or adding weights (top-p) per digit.
#include "aiq_internal.h"
#include "dev_util.h"

namespace aiq {

constexpr int SN = 1024;              // threads
constexpr int SW = SN / 64;           // waves
constexpr int BINS = 2048;

template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i) {
  if (DT == AIQ_F32) return static_cast<const float*>(p)[i];
  const uint16_t v = static_cast<const uint16_t*>(p)[i];
  return DT == AIQ_F16 ? h2f(v) : bf2f(v);
}

// Bit pattern that orders as the values (0 for NaN: below -infinity; -0 as 0)
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0;
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;   // order_key(-infinity)

struct Weigh {
  double inv_t, up, min_p;
  float m;
  // exp((x - m) / T); 1 at the maximum (an infinite one too), 0 for NaN and -infinity
  __device__ __forceinline__ double exp_of(float x) const {
    if (x == m) return 1.0;
    const double z = (static_cast<double>(x) - static_cast<double>(m)) * inv_t;
    return z > -700.0 ? exp(z) : 0.0;   // false for NaN
  }
  __device__ __forceinline__ uint64_t of(float x) const { return static_cast<uint64_t>(exp_of(x) * up + 0.5); }
  __device__ __forceinline__ uint64_t kept(float x) const {   // 0 below min_p
    const double e = exp_of(x);
    return e >= min_p ? static_cast<uint64_t>(e * up + 0.5) : 0;
  }
};

__device__ __forceinline__ uint64_t shfl_u64(uint64_t v, int mask) {
  const uint32_t lo = __shfl_xor(static_cast<uint32_t>(v), mask), hi = __shfl_xor(static_cast<uint32_t>(v >> 32), mask);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += shfl_u64(v, o);
  return v;
}
// inclusive sum over the lanes up to this one
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t lo = __shfl_up(static_cast<uint32_t>(v), o), hi = __shfl_up(static_cast<uint32_t>(v >> 32), o);
    if (lane >= o) v += (static_cast<uint64_t>(hi) << 32) | lo;
  }
  return v;
}

struct SampleLds {
  uint32_t cnt[BINS];
  uint64_t mass[BINS];
  uint64_t wave[SW];
  uint64_t before;
  uint32_t key, ties;
  int32_t id;
  uint32_t best;
};

// Sum of v over the workgroup, in every thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t v, SampleLds& s) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t t = 0;
#pragma unroll
  for (int w = 0; w < SW; ++w) t += s.wave[w];
  return t;
}

// The first token, in descending order, at which the count (MASS: the sum of
// weights) of the tokens so far reaches `target` (>= 1, at most all of it): its key
// in s.key and how many of the tokens with that key that takes in s.ties, the
// weights of those above the key in s.before.
template <int DT, bool MASS>
__device__ void find_prefix(const void* row, int V, const Weigh& w, uint64_t target, SampleLds& s) {
  const int tid = threadIdx.x, lane = tid & 63;
  uint32_t prefix = 0, mask = 0;
  uint64_t count_above = 0, mass_above = 0;
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0;
    const int bins = level == 2 ? 1024 : 2048;
    for (int b = tid; b < BINS; b += SN) {
      s.cnt[b] = 0;
      s.mass[b] = 0;
    }
    __syncthreads();
  #pragma unroll 2
    for (int i = tid; i < V; i += SN) {
      const float x = logit<DT>(row, i);
      const uint32_t k = order_key(x);
      if (k <= KEY_NEG_INF || (k & mask) != prefix) continue;
      const int b = (k >> shift) & (bins - 1);
      atomicAdd(&s.cnt[b], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[b]), static_cast<unsigned long long>(w.of(x)));
    }
    __syncthreads();
    // from the top: one wave, 64 runs of bins / 64 bins
    if (tid < 64) {
      const int per = bins / 64, top = bins - 1 - lane * per;
      uint64_t c = 0, ms = 0;
      for (int q = 0; q < per; ++q) {
        c += s.cnt[top - q];
        ms += s.mass[top - q];
      }
      const uint64_t ci = wave_scan_u64(c, lane), mi = wave_scan_u64(ms, lane);
      const uint64_t done = MASS ? mass_above + mi : count_above + ci;
      const uint64_t hit = __ballot(done >= target);
      if (hit && lane == __builtin_ctzll(hit)) {
        uint64_t ca = count_above + ci - c, ma = mass_above + mi - ms;
        int b = top;
        for (; b > top - per + 1; --b) {
          if ((MASS ? ma + s.mass[b] : ca + s.cnt[b]) >= target) break;
          ca += s.cnt[b];
          ma += s.mass[b];
        }
        s.key = prefix | (static_cast<uint32_t>(b) << shift);
        s.before = ma;
        s.wave[0] = ca;
        s.wave[1] = s.mass[b];
        s.wave[2] = s.cnt[b];
      }
    }
    __syncthreads();
    prefix = s.key;
    mask = shift ? ~((1u << shift) - 1u) : ~0u;
    mass_above = s.before;
    count_above = s.wave[0];
    if (level == 2 && tid == 0) {
      const uint64_t each = s.wave[1] / s.wave[2];   // equal logits, equal weights
      s.ties = static_cast<uint32_t>(MASS ? (target - mass_above + each - 1) / each : target - count_above);
    }
    __syncthreads();
  }
}

template <int DT>
__global__ __launch_bounds__(SN) void k_sample(SampleArgs a) {
  __shared__ SampleLds s;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int V = a.vocab;
  int64_t rows = a.n_rows;
  if (a.n_ptr && *a.n_ptr < rows) rows = *a.n_ptr;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const char* row = static_cast<const char*>(a.logits) + r * a.ld * (DT == AIQ_F32 ? 4 : 2);
    // the maximum, and the lowest id that has it
    uint64_t best = 0;   // (key, ~id)
    for (int i = tid; i < V; i += SN) {
      const uint64_t k = (static_cast<uint64_t>(order_key(logit<DT>(row, i))) << 32) | static_cast<uint32_t>(~i);
      best = k > best ? k : best;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t y = shfl_u64(best, o);
      best = y > best ? y : best;
    }
    __syncthreads();
    if (lane == 0) s.wave[wv] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SW; ++w) best = s.wave[w] > best ? s.wave[w] : best;
    __syncthreads();
    const uint32_t mk = static_cast<uint32_t>(best >> 32);
    const int first = static_cast<int>(~static_cast<uint32_t>(best));
    if (mk <= KEY_NEG_INF || a.temperature == 0.0) {
      if (tid == 0) a.token[r] = mk <= KEY_NEG_INF ? 0 : first;
      continue;
    }
    Weigh w;
    w.m = __uint_as_float(mk & 0x80000000u ? mk & 0x7FFFFFFFu : ~mk);
    w.inv_t = 1.0 / a.temperature;
    w.min_p = a.min_p;
    w.up = static_cast<double>(1ull << (62 - (32 - __builtin_clz(static_cast<uint32_t>(V)))));
    // the kept prefix: keys above `key`, and those equal to it up to id `last`
    uint32_t key = KEY_NEG_INF + 1;
    int last = V;
    uint32_t ties = 0;   // 0: all tokens equal to the key
    if (a.top_k > 0) {
      // fewer finite tokens than top_k: all of them
      uint32_t c = 0;
      for (int i = tid; i < V; i += SN) c += order_key(logit<DT>(row, i)) > KEY_NEG_INF;
      const uint64_t n = block_sum(c, s);
      if (n > static_cast<uint64_t>(a.top_k)) {
        find_prefix<DT, false>(row, V, w, a.top_k, s);
        key = s.key;
        ties = s.ties;
        __syncthreads();
      }
    }
    if (a.top_p < 1.0) {
      // the mass of the first n_k: keys above, and `ties` of the equal ones
      uint64_t above = 0;
      for (int i = tid; i < V; i += SN) {
        const float x = logit<DT>(row, i);
        const uint32_t k = order_key(x);
        if (k > key || (k == key && !ties)) above += w.of(x);
      }
      above = block_sum(above, s);
      if (ties) above += ties * w.of(__uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key));
      const double t = ceil(a.top_p * static_cast<double>(above));
      uint64_t target = t < 1.0 ? 1 : static_cast<uint64_t>(t);
      if (target > above) target = above;
      find_prefix<DT, true>(row, V, w, target, s);
      key = s.key;
      ties = s.ties;
      __syncthreads();
    }
    if (ties) {   // the id of the last of the equal tokens that belong: runs of V / SN ids per thread
      const int per = (V + SN - 1) / SN, i0 = tid * per, i1 = i0 + per < V ? i0 + per : V;
      uint32_t c = 0;
      for (int i = i0; i < i1; ++i) c += order_key(logit<DT>(row, i)) == key;
      const uint64_t incl = wave_scan_u64(c, lane);
      if (lane == 63) s.wave[wv] = incl;
      if (tid == 0) s.id = V;
      __syncthreads();
      uint64_t at = incl - c;
      for (int x = 0; x < wv; ++x) at += s.wave[x];
      if (c && at < ties && at + c >= ties)
        for (int i = i0; i < i1; ++i)
          if (order_key(logit<DT>(row, i)) == key && ++at == ties) s.id = i;
      __syncthreads();
      last = s.id;
      __syncthreads();
    }
    auto kept = [&](int i) -> uint64_t {
      if (i >= V) return 0;
      const float x = logit<DT>(row, i);
      const uint32_t k = order_key(x);
      return k > key || (k == key && i <= last) ? w.kept(x) : 0;
    };
    // each wave a run of ids; then the wave, then the 64 ids, that the random number falls into
    const int run = (V + SW * 64 - 1) / (SW * 64) * 64, i0 = wv * run;
    uint64_t mine = 0;
#pragma unroll 2
    for (int i = lane; i < run; i += 64) mine += kept(i0 + i);
    mine = wave_sum_u64(mine);
    if (lane == 0) s.wave[wv] = mine;
    __syncthreads();
    uint64_t total = 0;
#pragma unroll
    for (int x = 0; x < SW; ++x) total += s.wave[x];
    const int64_t ui = a.u_row ? a.u_row[*a.u_base + a.u_add + r] * a.u_ld + a.u_at : r;
    const double f = static_cast<double>(a.u[ui]);
    uint64_t target = total - 1;   // at least 1 kept: the maximum
    if (f < 1.0) {
      const double t = f * static_cast<double>(total);
      target = t > 0.0 ? static_cast<uint64_t>(t) : 0;
      if (target > total - 1) target = total - 1;
    }
    uint64_t at = 0;
    for (int x = 0; x < wv; ++x) at += s.wave[x];
    if (target >= at && target - at < mine) {   // this wave's
      for (int i = 0; i < run; i += 64) {
        const uint64_t incl = at + wave_scan_u64(kept(i0 + i + lane), lane);
        const uint64_t hit = __ballot(incl > target);
        if (hit) {
          if (lane == 0) a.token[r] = i0 + i + static_cast<int>(__builtin_ctzll(hit));
          break;
        }
        at = (static_cast<uint64_t>(__shfl(static_cast<uint32_t>(incl >> 32), 63)) << 32) | __shfl(static_cast<uint32_t>(incl), 63);
      }
    }
    __syncthreads();
  }
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(a.n_rows < 65536 ? a.n_rows : 65536));
  if (a.dtype == AIQ_F32)
    hipLaunchKernelGGL((k_sample<AIQ_F32>), grid, dim3(SN), 0, s, a);
  else if (a.dtype == AIQ_F16)
    hipLaunchKernelGGL((k_sample<AIQ_F16>), grid, dim3(SN), 0, s, a);
  else if (a.dtype == AIQ_BF16)
    hipLaunchKernelGGL((k_sample<AIQ_BF16>), grid, dim3(SN), 0, s, a);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace aiq
