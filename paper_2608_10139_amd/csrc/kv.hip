// Keys and values in 8 bits (Table 1's AI_TRANSFORM: the cache that a
// generation step writes and reads): quantising rows as they are written,
// reading them back, and attention over the cache.
//
// A block holds 32 tokens; per K/V head its keys and its values are bytes
// u = q + 128 with one fp32 scale each.  Inside a block the bytes lie in the
// order in which the attention's matrix instructions take them, so that a wave
// reads a block in whole 1 KB loads, 16 bytes per lane:
//   keys    token t, dim d: tile t / 16, 64-dim slice d / 64; lane (d % 64 / 16) * 16 + t % 16,
//           byte d % 16.  S^T = K Q^T on v_mfma_f32_16x16x32_f16 takes 8 dims of a lane per step.
//   values  token t, dim d: pair of 16-dim tiles d / 32; lane (t % 16 / 4) * 16 + d % 16,
//           byte (d % 32 / 16) * 8 + (t / 16) * 4 + t % 4.  S^T leaves, per lane, the scores of
//           4 tokens of each 16-token tile of one query: with the values' tokens in the same
//           order the weights are the operand of O^T = V^T P^T as they stand.
// The tail (16 bits) is plain rows.
#include "aiq_internal.h"
#include "dev_util.h"

#include <type_traits>

namespace aiq {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
typedef __attribute__((address_space(3))) uint16_t lds_u16;

constexpr int KVB = AIQ_KV_BLOCK;

// ------------------------------------------------------------------ sequences of a batch
struct KvSeq {
  int len, n;       // tokens in the cache, the call's rows among them
  int64_t row0;     // first row of the call
  int bs;           // first entry of its blocks
  int tail;
};

// a value that is the same for all lanes, in a scalar register (the compiler cannot know it of one read from memory)
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ void kv_flag(const KvBatch& b) {
  if (b.status) atomicOr(reinterpret_cast<unsigned long long*>(b.status), static_cast<unsigned long long>(AIQ_DEV_KV_RANGE));
}

// A sequence's numbers as they are in memory: read where they are used, or all at once.
struct KvAt {
  const KvBatch& b;
  int i;
  __device__ __forceinline__ int len() const { return b.len[i]; }
  __device__ __forceinline__ int c0() const { return b.cu[i]; }
  __device__ __forceinline__ int c1() const { return b.cu[i + 1]; }
  __device__ __forceinline__ int e0() const { return b.blk_start[i]; }
  __device__ __forceinline__ int e1() const { return b.blk_start[i + 1]; }
  __device__ __forceinline__ int tail() const { return b.tail_ids ? b.tail_ids[i] : i; }
};
struct KvRaw {   // of a batch with cu
  int v[6];
  __device__ __forceinline__ int len() const { return v[0]; }
  __device__ __forceinline__ int c0() const { return v[1]; }
  __device__ __forceinline__ int c1() const { return v[2]; }
  __device__ __forceinline__ int e0() const { return v[3]; }
  __device__ __forceinline__ int e1() const { return v[4]; }
  __device__ __forceinline__ int tail() const { return v[5]; }
};
// The sequence (i where there is no cu), or false where it is left out (its numbers do not fit, flagged; or it has no
// rows in this call).
template <typename S>
__device__ __forceinline__ bool kv_seq(const KvCache& c, const KvBatch& b, const S& r, int i, KvSeq& s) {
  s.len = uniform(r.len()) + b.len_add;
  if (b.cu) {
    const int c0 = uniform(r.c0()), c1 = uniform(r.c1());
    s.row0 = c0;
    s.n = c1 - c0 + b.n_pre;
    if (c0 < 0 || c1 < c0 || c1 > b.n_rows) {
      kv_flag(b);
      return false;
    }
  } else {
    s.row0 = i;
    s.n = s.len == 0 ? 0 : 1;
  }
  if (s.n == 0) return false;
  const int64_t e0 = uniform(r.e0()), e1 = uniform(r.e1());
  s.bs = static_cast<int>(e0);
  s.tail = uniform(r.tail());
  const bool uses_tail = s.len % KVB != 0 || (s.len - s.n) % KVB != 0;
  if (s.len < s.n || s.len > b.max_len || e0 < 0 || (c.n_blocks == 0 && s.len >= KVB) || (e1 - e0) * KVB < s.len ||
      e0 + s.len / KVB > b.n_ids || (uses_tail && (s.tail < 0 || s.tail >= c.n_tails))) {
    kv_flag(b);
    return false;
  }
  return true;
}

// Block number of entry e (of a full block of a sequence that kv_seq has let through), or -1 (flagged) where it is outside the cache.
__device__ __forceinline__ int kv_block(const KvCache& c, const KvBatch& b, int e) {
  const int id = b.blk_ids ? b.blk_ids[e] : e;
  if (id >= 0 && id < c.n_blocks) return id;
  kv_flag(b);
  return -1;
}

__device__ __forceinline__ int kv_count(const KvBatch& b) {
  if (!b.n_ptr) return b.n_seq;
  const int64_t n = uniform(static_cast<int>(*b.n_ptr));
  return n < b.n_seq ? static_cast<int>(n) : b.n_seq;
}

// Batches with several rows per sequence: sequence i owns the work units from
// first(i) = per * cu[i] / R + extra * i on, enough for `extra` + its rows / R
// units; which of them it fills the unit finds out itself.
__device__ __forceinline__ int64_t unit_first(const KvBatch& b, int i, int at, int per, int R, int extra) {   // at: cu[i]
  const int64_t c = (at < 0 ? 0 : at) + static_cast<int64_t>(i) * b.n_pre;
  return c * per / R + static_cast<int64_t>(extra) * i;
}
__device__ __forceinline__ int64_t unit_first(const KvBatch& b, int i, int per, int R, int extra) {
  return unit_first(b, i, uniform(b.cu[i]), per, R, extra);
}
// The last i with first(i) <= u (the same u for the wave's lanes): 64 places at a time, two rounds of reads
// for 4,096 sequences where halving takes twelve.
__device__ __forceinline__ int unit_seq(const KvBatch& b, int n, int64_t u, int per, int R, int extra) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const bool yes = i < hi && unit_first(b, i, b.cu[i < hi ? i : lo], per, R, extra) <= u;
    const uint64_t past = __ballot(yes);   // (first(lo) <= u: lane 0's at least, where cu is in order)
    const int k = past ? 63 - __builtin_clzll(past) : 0;
    lo += k * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return lo;
}

// ------------------------------------------------------------------ write and read
// A wave per (32-token block of a sequence that the call touches, K/V head);
// heads of a block are neighbours, so rows are read whole between them.
// Bound: HBM (2 bytes per element in, 1 out for full blocks; 2 out for the tail).  24/8 heads of 128: 1,500 prompts
// of about 120 tokens written in 332 us (1.35 GB, 4.1 TB/s) and read back in 262 (1.34 GB, 5.1 TB/s; a copy
// reaches 4.8); 2,000 whole sequences read in 61.
// The wave of a sequence's first touched block reads what the tail holds of
// it, and then writes the new tail: no other wave touches the tail.

// 4 values of one token as loaded: |x| as 16-bit patterns order like the values (infinity and NaN above all)
__device__ __forceinline__ uint32_t abs_max(uint32_t m, uint32_t two) {
  const uint32_t a = two & 0x7FFF7FFFu;
  const uint32_t lo = (a & 0xFFFFu) > (m & 0xFFFFu) ? (a & 0xFFFFu) : (m & 0xFFFFu);
  const uint32_t hi = (a >> 16) > (m >> 16) ? (a >> 16) : (m >> 16);
  return lo | (hi << 16);
}

// the block's scale and the nearest fp32 of 1 / scale
__device__ __forceinline__ float block_scale(uint32_t m, int act, float& inv) {
  uint32_t x = (m & 0xFFFFu) > (m >> 16) ? (m & 0xFFFFu) : (m >> 16);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t y = __shfl_xor(x, o);
    x = y > x ? y : x;
  }
  const uint32_t inf = act == ACT_F16 ? 0x7C00u : 0x7F80u;
  if (x >= inf) {
    inv = 0.f;
    return __uint_as_float(0x7FC00000u);
  }
  const float s = fmaxf(act2f(static_cast<uint16_t>(x), act), 0x1p-80f) / 127.0f;
  inv = 1.0f / s;
  return s;
}

// x / scale correctly rounded (quotient, exact remainder, one correction), rounded to a whole
// number by the add, in the low byte with 128 added.
__device__ __forceinline__ uint32_t quant(float x, float s, float inv) {
  const float q = x * inv;
  const float y = fmaf(fmaf(-q, s, x), inv, q);
  return __float_as_uint(y + (12582912.0f + 128.0f));   // 1.5 * 2^23
}
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return (a & 0xFFu) | ((b & 0xFFu) << 8) | ((c & 0xFFu) << 16) | (d << 24);
}

struct KvMoveArgs {
  KvCache c;
  KvBatch b;
  KvRows r;
};

// entry of the tail: keys (0) or values (1) of K/V head h
__device__ __forceinline__ uint16_t* tail_at(const KvCache& c, int tail, int kv, int h) {
  return c.tail + ((static_cast<int64_t>(tail) * 2 + kv) * c.n_kv + h) * (KVB * c.hd);
}

// work units of a batch: blocks that its rows touch (bound on the host, at most that on the device)
static __host__ __device__ int64_t move_units(const KvBatch& b) {
  return b.cu ? (b.n_rows + static_cast<int64_t>(b.n_seq) * b.n_pre) / KVB + 2 * static_cast<int64_t>(b.n_seq) : b.n_seq;
}
__device__ __forceinline__ int64_t move_count(const KvBatch& b, int n) {
  const int64_t u = b.cu ? unit_first(b, n, 1, KVB, 2) : n, ub = move_units(b);
  return u < ub ? u : ub;
}

// The unit's sequence and block; false: nothing to do.
__device__ __forceinline__ bool move_unit(const KvCache& c, const KvBatch& b, int n, int64_t u, KvSeq& s, int& jj) {
  int i = static_cast<int>(u);
  jj = 0;
  if (b.cu) {
    i = unit_seq(b, n, u, 1, KVB, 2);
    const int64_t d = u - unit_first(b, i, 1, KVB, 2);
    if (d < 0) return false;   // rows before the first sequence's
    jj = static_cast<int>(d);
  }
  return kv_seq(c, b, KvAt{b, i}, i, s);
}

// Block `id` of head h from its 32 tokens, the first one at position p0: those below `before` from the tail (tk, tv),
// the others from the rows that row_k and row_v give.
template <int HD, typename K, typename V>
__device__ __forceinline__ void write_block(const KvCache& c, int id, int h, int p0, int before, const uint16_t* tk, const uint16_t* tv,
                                            K row_k, V row_v) {
  constexpr int KC = HD / 64;
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
  const int64_t at = static_cast<int64_t>(id) * c.n_kv + h;
  uint4 kr[2 * KC][2];
  uint32_t m = 0;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = tt * 16 + c16, at_p = p0 + t;
    const uint16_t* p = (at_p < before ? tk + t * HD : row_k(at_p)) + g * 16;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int e = 0; e < 2; ++e) kr[tt * KC + kc][e] = *reinterpret_cast<const uint4*>(p + kc * 64 + e * 8);
  }
  uint2 vr[KC][2][4];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = tt * 16 + g * 4 + r, at_p = p0 + t;
      const uint16_t* p = (at_p < before ? tv + t * HD : row_v(at_p)) + c16 * 4;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) vr[kc][tt][r] = *reinterpret_cast<const uint2*>(p + kc * 64);
    }
#pragma unroll
  for (int i = 0; i < 2 * KC; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      m = abs_max(abs_max(abs_max(abs_max(m, kr[i][e].x), kr[i][e].y), kr[i][e].z), kr[i][e].w);
  float inv;
  float sc = block_scale(m, c.act, inv);
  if (lane == 0) c.ks[at] = sc;
  uint8_t* kb = c.k + at * (KVB * HD);
#pragma unroll
  for (int i = 0; i < 2 * KC; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t x[4] = {kr[i][e].x, kr[i][e].y, kr[i][e].z, kr[i][e].w};
      uint32_t b[8];
#pragma unroll
      for (int z = 0; z < 8; ++z)
        b[z] = quant(act2f(static_cast<uint16_t>(z & 1 ? x[z / 2] >> 16 : x[z / 2] & 0xFFFFu), c.act), sc, inv);
      w[e * 2] = pack4(b[0], b[1], b[2], b[3]);
      w[e * 2 + 1] = pack4(b[4], b[5], b[6], b[7]);
    }
    *reinterpret_cast<uint4*>(kb + (i * 64 + lane) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  m = 0;
#pragma unroll
  for (int kc = 0; kc < KC; ++kc)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = abs_max(abs_max(m, vr[kc][tt][r].x), vr[kc][tt][r].y);
  sc = block_scale(m, c.act, inv);
  if (lane == 0) c.vs[at] = sc;
  uint8_t* vb = c.v + at * (KVB * HD);
#pragma unroll
  for (int kc = 0; kc < KC; ++kc)
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const int d = kc * 64 + c16 * 4 + z;   // its 8 tokens of this lane group
      uint32_t w[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        uint32_t b[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t x = z < 2 ? vr[kc][tt][r].x : vr[kc][tt][r].y;
          b[r] = quant(act2f(static_cast<uint16_t>(z & 1 ? x >> 16 : x & 0xFFFFu), c.act), sc, inv);
        }
        w[tt] = pack4(b[0], b[1], b[2], b[3]);
      }
      *reinterpret_cast<uint2*>(vb + ((d / 32) * 64 + g * 16 + d % 16) * 16 + (d % 32 / 16) * 8) =
          make_uint2(w[0], w[1]);
    }
}

template <int HD>
__global__ __launch_bounds__(256) void k_kv_write(KvMoveArgs a) {
  const KvCache& c = a.c;
  const int n = kv_count(a.b);
  if (n <= 0) return;
  const int lane = threadIdx.x & 63;
  const int64_t units = move_count(a.b, n);
  const int64_t wave = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) >> 6;
  const int64_t n_waves = (static_cast<int64_t>(gridDim.x) * blockDim.x) >> 6;
  for (int64_t item = wave; item < units * c.n_kv; item += n_waves) {
    const int64_t u = uniform(static_cast<int>(item / c.n_kv));   // (units are below 2^31)
    const int h = uniform(static_cast<int>(item - u * c.n_kv));
    KvSeq s;
    int jj;
    if (!move_unit(c, a.b, n, u, s, jj)) continue;
    const int before = s.len - s.n;
    const int j = before / KVB + jj;
    if (j * KVB >= s.len) continue;
    uint16_t* tk = tail_at(c, s.tail, 0, h);
    uint16_t* tv = tail_at(c, s.tail, 1, h);
    // rows of token p, not in the cache before this call
    auto row_k = [&](int p) {
      const int64_t r = p - before;
      return (r < a.b.n_pre ? a.r.pk + r * a.r.k_ld : a.r.k + (s.row0 + r - a.b.n_pre) * a.r.k_ld) + h * HD;
    };
    auto row_v = [&](int p) {
      const int64_t r = p - before;
      return (r < a.b.n_pre ? a.r.pv + r * a.r.v_ld : a.r.v + (s.row0 + r - a.b.n_pre) * a.r.v_ld) + h * HD;
    };
    if ((j + 1) * KVB <= s.len) {
      const int id = kv_block(c, a.b, s.bs + j);
      if (id >= 0) write_block<HD>(c, id, h, j * KVB, before, tk, tv, row_k, row_v);
    }
    if (jj != 0 || s.len % KVB == 0) continue;
    // the tail: the new tokens of the last block, after this wave's own reads of the old one
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    const int t0 = s.len / KVB * KVB > before ? s.len / KVB * KVB : before;
    for (int x = lane; x < (s.len - t0) * (HD / 8); x += 64) {
      const int t = t0 + x / (HD / 8), e = x % (HD / 8) * 8;
      *reinterpret_cast<uint4*>(tk + t % KVB * HD + e) = *reinterpret_cast<const uint4*>(row_k(t) + e);
      *reinterpret_cast<uint4*>(tv + t % KVB * HD + e) = *reinterpret_cast<const uint4*>(row_v(t) + e);
    }
  }
}

// One row per sequence (no cu): a wave per sequence writes its row of all heads into the tail; the blocks that a
// workgroup's sequences complete, one in 32 steps, are then its eight waves', a head each at a time (4 us for one: cold
// loads, then the rounding).  A workgroup takes up to eight sequences, fewer where that leaves CUs without any: 64
// that complete a block at once 55 us by eights, 13 by ones.  2,000 sequences of 24/8 heads of 128, a 32nd of them with a
// block complete, 20 us where a wave per (sequence, head) took 23; a query of 16,384 rows with 128 steps of 4 layers
// 720 ms for 753.
template <int HD>
__global__ __launch_bounds__(512) void k_kv_write_one(KvMoveArgs a, int per) {
  __shared__ int full[8][3];   // of the sequences that complete a block: its number, its first token, the tail
  const KvCache& c = a.c;
  const int n = kv_count(a.b);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int i0 = blockIdx.x * per; i0 < n; i0 += gridDim.x * per) {
    KvSeq s;
    const bool is = w < per && i0 + w < n && kv_seq(c, a.b, KvAt{a.b, i0 + w}, i0 + w, s);
    const int id = is && s.len % KVB == 0 ? kv_block(c, a.b, s.bs + s.len / KVB - 1) : -1;
    if (lane == 0) {
      full[w][0] = id;
      full[w][1] = id < 0 ? 0 : s.len - KVB;
      full[w][2] = id < 0 ? 0 : s.tail;
    }
    if (is && s.len % KVB != 0) {
      const int t = s.len % KVB - 1, pieces = c.n_kv * (HD / 8);
      const uint16_t* k = a.r.k + s.row0 * a.r.k_ld;
      const uint16_t* v = a.r.v + s.row0 * a.r.v_ld;
      uint16_t* tk = tail_at(c, s.tail, 0, 0) + t * HD;
      uint16_t* tv = tail_at(c, s.tail, 1, 0) + t * HD;
      auto to = [](int x) { return x / (HD / 8) * static_cast<int64_t>(KVB * HD) + x % (HD / 8) * 8; };
      for (int x = lane; x < pieces; x += 128) {
        const int y = x + 64 < pieces ? x + 64 : x;
        const uint4 kx = *reinterpret_cast<const uint4*>(k + x * 8), vx = *reinterpret_cast<const uint4*>(v + x * 8);
        const uint4 ky = *reinterpret_cast<const uint4*>(k + y * 8), vy = *reinterpret_cast<const uint4*>(v + y * 8);
        *reinterpret_cast<uint4*>(tk + to(x)) = kx;
        *reinterpret_cast<uint4*>(tv + to(x)) = vx;
        *reinterpret_cast<uint4*>(tk + to(y)) = ky;
        *reinterpret_cast<uint4*>(tv + to(y)) = vy;
      }
    }
    __syncthreads();
    for (int q = 0; q < per; ++q) {
      const int bid = uniform(full[q][0]), p0 = uniform(full[q][1]), tail = uniform(full[q][2]);
      if (bid < 0) continue;
      for (int h = w; h < c.n_kv; h += 8) {
        const uint16_t* k = a.r.k + (i0 + q) * a.r.k_ld + h * HD;
        const uint16_t* v = a.r.v + (i0 + q) * a.r.v_ld + h * HD;
        write_block<HD>(c, bid, h, p0, p0 + KVB - 1, tail_at(c, tail, 0, h), tail_at(c, tail, 1, h), [&](int) { return k; },
                        [&](int) { return v; });
      }
    }
    __syncthreads();
  }
}

// (u - 128) * scale in the cache's 16-bit type
__device__ __forceinline__ uint32_t unq(uint32_t word, int byte, float s, int act) {
  return f2act((static_cast<float>((word >> (8 * byte)) & 0xFFu) - 128.0f) * s, act);
}

template <int HD>
__global__ __launch_bounds__(256) void k_kv_read(KvMoveArgs a) {
  constexpr int KC = HD / 64;
  const KvCache& c = a.c;
  const int n = kv_count(a.b);
  if (n <= 0) return;
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
  const int64_t units = move_count(a.b, n);
  const int64_t wave = (blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x) >> 6;
  const int64_t n_waves = (static_cast<int64_t>(gridDim.x) * blockDim.x) >> 6;
  for (int64_t item = wave; item < units * c.n_kv; item += n_waves) {
    const int64_t u = uniform(static_cast<int>(item / c.n_kv));   // (units are below 2^31)
    const int h = uniform(static_cast<int>(item - u * c.n_kv));
    KvSeq s;
    int jj;
    if (!move_unit(c, a.b, n, u, s, jj)) continue;
    const int before = s.len - s.n;
    const int j = before / KVB + jj;
    if (j * KVB >= s.len) continue;
    uint16_t* ko = a.r.k + s.row0 * a.r.k_ld + h * HD;   // row of token `before`
    uint16_t* vo = a.r.v + s.row0 * a.r.v_ld + h * HD;
    if ((j + 1) * KVB > s.len) {
      const uint16_t* tk = tail_at(c, s.tail, 0, h);
      const uint16_t* tv = tail_at(c, s.tail, 1, h);
      const int t0 = j * KVB > before ? j * KVB : before;
      const int pieces = (s.len - t0) * (HD / 8);
      for (int x0 = 0; x0 < pieces; x0 += 256) {   // four loads of keys and of values in flight
        auto from = [&](const uint16_t* t, int q) {
          const int x = x0 + q * 64 + lane < pieces ? x0 + q * 64 + lane : pieces - 1;
          return *reinterpret_cast<const uint4*>(t + (t0 + x / (HD / 8)) % KVB * HD + x % (HD / 8) * 8);
        };
        auto to = [&](int q, const uint4& kk, const uint4& vv) {
          const int x = x0 + q * 64 + lane, e = x % (HD / 8) * 8;
          const int64_t r = t0 + x / (HD / 8) - before;
          if (x >= pieces) return;
          *reinterpret_cast<uint4*>(ko + r * a.r.k_ld + e) = kk;
          *reinterpret_cast<uint4*>(vo + r * a.r.v_ld + e) = vv;
        };
        const uint4 k0 = from(tk, 0), k1 = from(tk, 1), k2 = from(tk, 2), k3 = from(tk, 3);
        const uint4 v0 = from(tv, 0), v1 = from(tv, 1), v2 = from(tv, 2), v3 = from(tv, 3);
        to(0, k0, v0);
        to(1, k1, v1);
        to(2, k2, v2);
        to(3, k3, v3);
      }
      continue;
    }
    const int id = kv_block(c, a.b, s.bs + j);
    if (id < 0) continue;
    const int64_t at = static_cast<int64_t>(id) * c.n_kv + h;
    const float ks = c.ks[at], vs = c.vs[at];
    const uint8_t* kb = c.k + at * (KVB * HD);
    const uint8_t* vb = c.v + at * (KVB * HD);
    uint4 kr[2 * KC];
#pragma unroll
    for (int i = 0; i < 2 * KC; ++i) kr[i] = *reinterpret_cast<const uint4*>(kb + (i * 64 + lane) * 16);
    uint2 vr[KC][4];
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const int d = kc * 64 + c16 * 4 + z;
        vr[kc][z] = *reinterpret_cast<const uint2*>(vb + ((d / 32) * 64 + g * 16 + d % 16) * 16 + (d % 32 / 16) * 8);
      }
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int r = j * KVB + tt * 16 + c16 - before;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        const uint32_t x[4] = {kr[tt * KC + kc].x, kr[tt * KC + kc].y, kr[tt * KC + kc].z, kr[tt * KC + kc].w};
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          w[e] = unq(x[e / 2], e % 2 * 2, ks, c.act) | (unq(x[e / 2], e % 2 * 2 + 1, ks, c.act) << 16);
        if (r < 0) continue;
        uint4* o = reinterpret_cast<uint4*>(ko + r * a.r.k_ld + kc * 64 + g * 16);
        o[0] = make_uint4(w[0], w[1], w[2], w[3]);
        o[1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int r = j * KVB + tt * 16 + g * 4 + r4 - before;
        if (r < 0) continue;
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          uint32_t w[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) w[z] = unq(tt ? vr[kc][z].y : vr[kc][z].x, r4, vs, c.act);
          *reinterpret_cast<uint2*>(vo + r * a.r.v_ld + kc * 64 + c16 * 4) =
              make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
        }
      }
  }
}

static int kv_grid(int64_t waves, int cap) {
  int64_t g = (waves + 3) / 4;
  if (g < 1) g = 1;
  return static_cast<int>(g > cap ? cap : g);
}

hipError_t launch_kv_write(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t s) {
  if (b.n_seq == 0 || (b.n_rows == 0 && b.n_pre == 0)) return hipSuccess;
  if (b.n_pre < 0 || (b.n_pre > 0 && (!b.cu || !r.pk || !r.pv))) return hipErrorInvalidValue;
  const KvMoveArgs a{c, b, r};
  // (with n_ptr a bound from the host only: the sequences may be few)
  const int cap = b.n_ptr ? 1 << 13 : 1 << 16, per = b.n_seq < 2048 ? (b.n_seq + 255) / 256 : 8;
  const dim3 grid(kv_grid(move_units(b) * c.n_kv, cap)), one(kv_grid((b.n_seq + per - 1) / per * static_cast<int64_t>(4), cap));
  if (c.hd == 64 && b.cu)
    hipLaunchKernelGGL((k_kv_write<64>), grid, dim3(256), 0, s, a);
  else if (c.hd == 64)
    hipLaunchKernelGGL((k_kv_write_one<64>), one, dim3(512), 0, s, a, per);
  else if (c.hd == 128 && b.cu)
    hipLaunchKernelGGL((k_kv_write<128>), grid, dim3(256), 0, s, a);
  else if (c.hd == 128)
    hipLaunchKernelGGL((k_kv_write_one<128>), one, dim3(512), 0, s, a, per);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void k_kv_plan(const int64_t* desc, const int64_t* cu, int32_t npre, int32_t gen,
                                                 int32_t n_ub, int32_t* plen, int32_t* cu32, int32_t* blk) {
  const int64_t sb = desc[D_SEQ_BEGIN], tb = desc[D_TOK_BEGIN], ns = desc[D_NSEQ];
  const int64_t n = ns < n_ub ? ns : n_ub;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i <= n;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t c = cu[sb + i] - tb;
    cu32[i] = static_cast<int32_t>(c);
    // room for ceil of a sequence's tokens / 32: floors of the running sums differ by its floor at least
    blk[i] = static_cast<int32_t>((c + i * (npre + gen)) / KVB + i);
    if (i < n) plen[i] = npre + static_cast<int32_t>(cu[sb + i + 1] - cu[sb + i]);
  }
}

hipError_t launch_kv_plan(const int64_t* desc, const int64_t* cu, int32_t npre, int32_t gen, int32_t n_ub,
                          int32_t* plen, int32_t* cu32, int32_t* blk, hipStream_t s) {
  const int64_t g = (static_cast<int64_t>(n_ub) + 256) / 256;
  hipLaunchKernelGGL(k_kv_plan, dim3(static_cast<unsigned>(g < 4096 ? g : 4096)), dim3(256), 0, s, desc, cu, npre, gen,
                     n_ub, plen, cu32, blk);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t s) {
  if (b.n_seq == 0 || b.n_rows == 0) return hipSuccess;
  const KvMoveArgs a{c, b, r};
  const dim3 grid(kv_grid(move_units(b) * c.n_kv, 1 << 16));
  if (c.hd == 64)
    hipLaunchKernelGGL((k_kv_read<64>), grid, dim3(256), 0, s, a);
  else if (c.hd == 128)
    hipLaunchKernelGGL((k_kv_read<128>), grid, dim3(256), 0, s, a);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

// ------------------------------------------------------------------ attention
// A tile is 16 query rows of a (sequence, K/V head): row r is query r / rep of
// the sequence's and head r % rep of the group, one per lane column.  A
// workgroup's four waves share a tile's keys in segments of 512 tokens: wave w
// takes blocks w, w + 4, .. of the segment, each with a softmax state of its
// own, folded in order at the segment's end and segment after segment.  The
// order depends on the keys alone, so with one row per sequence a sequence's
// bits do not depend on the batch, nor on whether its segments run in one
// workgroup or (SPLIT, few long sequences) in one each with the fold in a
// second launch.
// Per block: s' = log2(e) / sqrt(hd) * k_scale * (q . k_u) + log2(v_scale), the weights
// p' = 2^(s' - m) against a running reference m, numerator += p' v_u, denominator
// += sum p' / v_scale: a block's scales cost two multiply-adds per score, the
// bytes themselves (whole numbers, exact in fp16) go into the matrix products.
// m follows the maximum only when that is more than 8 above it (so weights
// stay below 2^8 and, with the fixed factor 2^7, in fp16's normal range down to 2^-21 of
// the largest at least).  fp16 holds the weights to 2^-11 relative, as the 16-bit attention does, and to 2^-25 below that
// range (2^-32 of the largest); their sums stay in 32 bits.  The tail of a bf16 cache has bf16 values and a product
// of that type: its weights are held to 2^-8 (the values may be past fp16's range).
// Bound: HBM, as every byte of the cache is read once: 2,000 sequences of about 200 tokens (24/8 heads of 128, waves
// alone) 224 us for 1.14 GB, 5.1 TB/s; 4 of 100,000 (32/8 heads of 64, split) 83 us for 417 MB, 5.0 TB/s; one of
// 171 tokens 6.5 us, the chain of one wave's loads and products; 256 of about 150 (8/8 heads of 64) 18 us for 52 MB, 2.8
// TB/s: the four waves take up to 127 registers, so that four workgroups are on a CU, 1,024 of the 2,048 at a time, and long
// sequences may start late.  These kernels keep 22 to 65 scalars in vector lanes; none of them spills to scratch.
constexpr int KV_SEG = 16;       // blocks per segment
constexpr float KV_SLACK = 8.0f, KV_UP = 7.0f;
constexpr int KV_MANY = 48;      // rows per sequence from which on tiles of KV_ROWS take them

__device__ __forceinline__ float swap_max(float v) {   // over the wave's four lane groups
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float swap_add(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// LDS written by a wave, read by the same wave
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 8 bytes u = q + 128 as the fp16 values q: 0x64uu is 1024 + u
__device__ __forceinline__ half8 bytes_f16(uint32_t lo, uint32_t hi) {
  union {
    uint32_t w[4];
    half8 h;
  } x;
  x.w[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
  x.w[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
  x.w[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
  x.w[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
  const half8 off = {1152, 1152, 1152, 1152, 1152, 1152, 1152, 1152};
  return x.h - off;
}

// bf16 query fragments (a row's in the lanes of one column) as fp16 times a power of two, exact but for values
// 2^-25 of the row's largest; returns the power that undoes it
template <int N>
__device__ __forceinline__ float rows_f16(half8 (&q)[N]) {
  float mx = 0.f;
#pragma unroll
  for (int x = 0; x < N; ++x) {
    const uint4 v = __builtin_bit_cast(uint4, q[x]);
    const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mx = fmaxf(mx, fabsf(__uint_as_float(y[e] << 16)));
      mx = fmaxf(mx, fabsf(__uint_as_float(y[e] & 0xFFFF0000u)));
    }
  }
  mx = swap_max(mx);
  int ex = static_cast<int>(__float_as_uint(mx) >> 23) - 127;   // mx in [2^ex, 2^(ex + 1))
  ex = ex < -100 ? -100 : ex;
  const float up = __uint_as_float(static_cast<uint32_t>(127 + 8 - ex) << 23);
#pragma unroll
  for (int x = 0; x < N; ++x) {
    const uint4 v = __builtin_bit_cast(uint4, q[x]);
    const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      q[x][2 * e] = static_cast<_Float16>(__uint_as_float(y[e] << 16) * up);
      q[x][2 * e + 1] = static_cast<_Float16>(__uint_as_float(y[e] & 0xFFFF0000u) * up);
    }
  }
  return __uint_as_float(static_cast<uint32_t>(127 - 8 + ex) << 23);
}

// What a block's scales make of its scores: times k, plus the log2 of the values' scale, and that
// inverted for the sums.  A block with an infinity or NaN has scores of NaN instead (bad), so that
// tokens that a row does not see can still be masked.  A values' scale below the least that is written (of a block that
// never was) counts as that one: its tokens weigh what their scores say.
struct KvScale {
  float k, log_v, inv_v;
  bool bad;
};
__device__ __forceinline__ KvScale kv_scale(float ks, float vs) {
  const bool bad = !(ks < INFINITY) || !(vs < INFINITY);
  vs = bad ? 1.f : fmaxf(vs, 0x1p-80f / 127.0f);
  return {bad ? 1.f : ks, __builtin_amdgcn_logf(vs), 1.0f / vs, bad};
}

// Scores of NaN for a block that holds one; -infinity for tokens (tok + 0 .. 3, tok + 16 .. 19) past pos.
__device__ __forceinline__ void kv_mask(f32x4 (&acc)[2], bool bad, bool masked, int tok, int pos) {
  if (__builtin_expect(bad, 0)) {
    asm volatile("");   // a branch, not selects for every block
    acc[0] = acc[1] = f32x4{NAN, NAN, NAN, NAN};
  }
  if (masked) {
    asm volatile("");
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (tok + (e / 4) * 16 + e % 4 > pos) acc[e / 4][e % 4] = -INFINITY;
  }
}

__device__ __forceinline__ float max3(float a, float b, float c) {   // (fmaxf would quiet its operands first)
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// The softmax of S blocks for T tiles of 16 rows, a row per lane column: from the scores acc of this
// lane's 8 tokens of each times c1 plus c2 the weights p, against the references m, which follow; the
// sums l and numerators o with them.
template <int S, int T, int NO>
__device__ __forceinline__ void kv_softmax(const f32x4 (&acc)[S][T][2], const float (&c1)[S][T], const float (&c2)[S],
                                           const float (&inv)[S], float (&m)[T], float (&l)[T], f32x4 (&o)[T][NO],
                                           float (&p)[S][T][8]) {
  float mx[T];
  bool up = false;
#pragma unroll
  for (int x = 0; x < T; ++x) {
    mx[x] = -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s) {   // (c1 > 0: the largest score is that of the largest product)
      const f32x4 a = acc[s][x][0], b = acc[s][x][1];
      mx[x] = fmaxf(mx[x], fmaf(max3(max3(a[0], a[1], a[2]), max3(a[3], b[0], b[1]), fmaxf(b[2], b[3])), c1[s][x], c2[s]));
    }
    up = up || mx[x] > m[x] + KV_SLACK;
  }
  if (__any(up)) {
#pragma unroll
    for (int x = 0; x < T; ++x) {
      const float mn = fmaxf(m[x], swap_max(mx[x]));
      const float al = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - mn);
#pragma unroll
      for (int y = 0; y < NO; ++y) o[x][y] *= al;
      l[x] *= al;
      m[x] = mn;
    }
  }
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int x = 0; x < T; ++x) {
      float (&w)[8] = p[s][x];
      const float off = c2[s] - (m[x] == -INFINITY ? 0.f : m[x] - KV_UP);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(acc[s][x][e / 4][e % 4], c1[s][x], off));
      const float ps = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
      l[x] = fmaf(ps, inv[s], l[x]);
    }
}
// a factor of scores: positive, so that the product with -infinity is that
__device__ __forceinline__ float kv_factor(float fac, float ks) { return fmaxf(fac * ks, 0x1p-126f); }

// 1 / sum of a row that sees nb blocks: 0 for an empty slot's, which sees none.  A sum of 0 over blocks comes of scores that
// are all -infinity (an infinite query): infinity, and not a number times the numerator of 0, as the formula has it.
__device__ __forceinline__ float kv_inverse(float l, int nb) { return nb == 0 ? 0.f : 1.0f / l; }

// softmax state of one row: reference, sum, one value of the numerator
__device__ __forceinline__ void kv_fold(float& m, float& l, float& o, float mp, float lp, float op) {
  const float mn = fmaxf(m, mp);
  const float ref = mn == -INFINITY ? 0.f : mn;
  const float x = __builtin_amdgcn_exp2f(m - ref), y = __builtin_amdgcn_exp2f(mp - ref);
  l = fmaf(lp, y, l * x);
  o = fmaf(op, y, o * x);
  m = mn;
}

struct KvTile {
  KvSeq s;
  int r0, rows;      // first row of the tile (of the sequence's n * rep), rows in it
  int nb;            // blocks that its last query sees
  int pos0;          // position of the tile's first query
};

// Tile u (of R rows) of the batch, or of the sequence whose numbers are given; or false
template <int R, typename S = int>
__device__ __forceinline__ bool kv_tile(const KvAttendArgs& a, int n, int rep, int64_t u, KvTile& t, const S* seq = nullptr) {
  int i = 0;
  int64_t k = u;
  if constexpr (!std::is_same_v<S, int>) {
    if (!kv_seq(a.c, a.b, *seq, 0, t.s)) return false;
  } else {
    if (a.b.cu) {
      i = unit_seq(a.b, n, u, rep, R, 1);
      k = u - unit_first(a.b, i, rep, R, 1);
    } else {
      const int tiles = (rep + 15) / 16;
      i = static_cast<int>(u / tiles);
      k = u - static_cast<int64_t>(i) * tiles;
    }
    if (!kv_seq(a.c, a.b, KvAt{a.b, i}, i, t.s)) {
      if (!a.b.cu && t.s.len == 0) {   // an empty slot's row
        t.r0 = static_cast<int>(k) * 16;
        t.rows = rep - t.r0 < 16 ? rep - t.r0 : 16;
        t.nb = 0;
        t.pos0 = 0;
        t.s.n = 1;
        return true;
      }
      return false;
    }
  }
  const int64_t all = static_cast<int64_t>(t.s.n) * rep;
  if (k < 0 || k * R >= all) return false;   // (k < 0: rows before the first sequence's)
  t.r0 = static_cast<int>(k * R);
  t.rows = static_cast<int>(all - t.r0 < R ? all - t.r0 : R);
  t.pos0 = t.s.len - t.s.n + t.r0 / rep;
  t.nb = (t.s.len - t.s.n + (t.r0 + t.rows - 1) / rep) / KVB + 1;
  return true;
}

// One wave's part of a tile: its queries, and the softmax state (m, l, o) of
// the blocks it has taken since reset().
template <int HD, bool BF, bool LEAN>
struct KvWave {
  static constexpr int KC = HD / 64, NO = HD / 16;
  const KvAttendArgs& a;
  const KvTile& t;
  uint16_t* vt;         // LDS: the tail's values, for transposing reads
  int* bad;             // LDS: its tokens with an infinity or NaN
  int h, lane, g, c16, pos;
  const uint16_t* qp;
  float fac;
  half8 qf[KC * 2];
  int id;               // lane x < KV_SEG: the segment's block x, its scales (a number out of bounds: block 0, its
  KvScale sc;           // tokens weigh nothing)

  uint4 kr[2 * KC];     // the next block's keys
  f32x4 o[1][NO];       // (one tile of kv_softmax)
  float m[1], l[1];

  __device__ __forceinline__ KvWave(const KvAttendArgs& a_, const KvTile& t_, int h_, int rep, uint16_t* vt_, int* bad_)
      : a(a_), t(t_), vt(vt_), bad(bad_), h(h_), lane(threadIdx.x & 63), g(lane >> 4), c16(lane & 15) {
    // queries: lane (g, c16) holds row c16, dims 64 kc + 16 g + 8 e .. + 7
    const int row = t.r0 + (c16 < t.rows ? c16 : 0);
    pos = t.s.len - t.s.n + row / rep;
    qp = a.q + (t.s.row0 + row / rep) * a.q_ld + (h * rep + row % rep) * HD + g * 16;
    fac = 1.4426950408889634f / sqrtf(static_cast<float>(HD));
#pragma unroll
    for (int x = 0; x < KC * 2; ++x)
      qf[x] = __builtin_bit_cast(half8, *reinterpret_cast<const uint4*>(qp + (x / 2) * 64 + (x % 2) * 8));
    if (BF) fac *= rows_f16<KC * 2>(qf);
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int x = 0; x < NO; ++x) o[0][x] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[0] = -INFINITY;
    l[0] = 0.f;
  }
  __device__ __forceinline__ void segment(int seg) {
    const int j = seg * KV_SEG + lane;
    id = 0;
    sc = {1.f, -INFINITY, 1.f, false};
    if (lane < KV_SEG && j < t.nb && (j + 1) * KVB <= t.s.len) {
      id = kv_block(a.c, a.b, t.s.bs + j);
      if (id >= 0) {
        const int64_t at = static_cast<int64_t>(id) * a.c.n_kv + h;
        sc = kv_scale(a.c.ks[at], a.c.vs[at]);
      }
      id = id < 0 ? 0 : id;
    }
  }
  // of the nbs blocks that the tile sees of a segment, those that are not the tail
  __device__ __forceinline__ int full_blocks(int seg, int nbs) const {
    const int f = t.s.len / KVB - seg * KV_SEG;
    return f < nbs ? f : nbs;
  }
  __device__ __forceinline__ int64_t at(int bid) const { return (static_cast<int64_t>(bid) * a.c.n_kv + h) * (KVB * HD); }
  // the keys of block k of the segment (a full one; k < 0: none)
  __device__ __forceinline__ void load(int k) {
    if (k < 0) return;
    const uint8_t* p = a.c.k + at(__builtin_amdgcn_readlane(id, k));
    const uint32_t off = static_cast<uint32_t>(lane) * 16;
#pragma unroll
    for (int x = 0; x < 2 * KC; ++x) kr[x] = *reinterpret_cast<const uint4*>(p + x * 1024 + off);
  }
  __device__ __forceinline__ void weigh(f32x4 (&acc)[1][1][2], float c1, float c2, float inv, bool no, int tok0, bool masked,
                                        float (&p)[1][1][8]) {
    const float f[1][1] = {{c1}}, add[1] = {c2}, over[1] = {inv};
    kv_mask(acc[0][0], no, masked, tok0 + g * 4, pos);
    kv_softmax<1, 1, NO>(acc, f, add, over, m, l, o, p);
  }
  // block k of the segment, whose keys load() has read; its values are read while its scores are
  // computed, the keys of block kn while its weights and values are
  __device__ __forceinline__ void take(int seg, int k, int kn) {
    const int tok0 = (seg * KV_SEG + k) * KVB;
    const int bid = __builtin_amdgcn_readlane(id, k);
    uint4 vr[2 * KC];
    const uint8_t* vp = a.c.v + at(bid);
    const uint32_t off = static_cast<uint32_t>(lane) * 16;
#pragma unroll
    for (int x = 0; x < 2 * KC; ++x) vr[x] = *reinterpret_cast<const uint4*>(vp + x * 1024 + off);
    auto of = [&](float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), k)); };
    f32x4 acc[1][1][2] = {{{f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}}};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const uint4 y = kr[tt * KC + kc];
        acc[0][0][tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bytes_f16(y.x, y.y), qf[kc * 2], acc[0][0][tt], 0, 0, 0);
        acc[0][0][tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bytes_f16(y.z, y.w), qf[kc * 2 + 1], acc[0][0][tt], 0, 0, 0);
      }
    load(kn);
    float p[1][1][8];
    weigh(acc, kv_factor(fac, of(sc.k)), of(sc.log_v), of(sc.inv_v), __builtin_amdgcn_readlane(sc.bad, k) != 0, tok0, tok0 + KVB - 1 > t.pos0, p);
    half8 pf;
#pragma unroll
    for (int e = 0; e < 8; ++e) pf[e] = static_cast<_Float16>(p[0][0][e]);
#pragma unroll
    for (int x = 0; x < 2 * KC; ++x) {
      o[0][2 * x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bytes_f16(vr[x].x, vr[x].y), pf, o[0][2 * x], 0, 0, 0);
      o[0][2 * x + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bytes_f16(vr[x].z, vr[x].w), pf, o[0][2 * x + 1], 0, 0, 0);
    }
  }
  // the tail: 16-bit rows, products in their own type; rows past the length are read as the last one, and
  // zeroed where that matters.  Values go through LDS, row-major, in 16-byte pieces (swizzled by the row).
  __device__ __forceinline__ void tail(int tok0) {
    const int left = t.s.len - tok0;
    // (its addresses are not worth registers through the whole loop: computed here)
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int g = ln >> 4, c16 = ln & 15;
    const uint16_t* tk = tail_at(a.c, t.s.tail, 0, h);
    const uint16_t* tv = tail_at(a.c, t.s.tail, 1, h);
    const bool several = a.b.cu != nullptr;
    constexpr int PIECES = HD / 8, PER = KVB * PIECES / 64;
    uint4 kt[4 * KC], vv[PER];
    f32x4 acc[1][1][2] = {{{f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}}};
    auto load_keys = [&]() {
#pragma unroll
      for (int x = 0; x < 4 * KC; ++x) {   // token x / (2 KC) * 16 + c16
        const int tok = (x / (2 * KC)) * 16 + c16, row = tok < left ? tok : left - 1;
        kt[x] = *reinterpret_cast<const uint4*>(tk + static_cast<uint32_t>(row * HD + (x % (2 * KC) / 2) * 64 + g * 16 + (x % 2) * 8));
      }
    };
    if (!LEAN) load_keys();
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int tok = (x * 64 + ln) / PIECES, row = tok < left ? tok : left - 1;
      vv[x] = *reinterpret_cast<const uint4*>(tv + static_cast<uint32_t>(row * HD + (x * 64 + ln) % PIECES * 8));
    }
    if (several) bad[ln & (KVB - 1)] = 0;
    wave_sync();
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int tok = (x * 64 + ln) / PIECES, ch = (x * 64 + ln) % PIECES;
      uint4 y = vv[x];
      bool none = tok >= left;
      if (several) {   // a later query's infinity or NaN must not meet the weight 0
        const uint32_t z = abs_max(abs_max(abs_max(abs_max(0, y.x), y.y), y.z), y.w), inf = BF ? 0x7F80u : 0x7C00u;
        if (!none && ((z & 0xFFFFu) >= inf || (z >> 16) >= inf)) {
          none = true;
          bad[tok] = 1;
        }
      }
      y.x = none ? 0 : y.x;
      y.y = none ? 0 : y.y;
      y.z = none ? 0 : y.z;
      y.w = none ? 0 : y.w;
      *reinterpret_cast<uint4*>(vt + tok * HD + ((ch ^ (tok & 7)) << 3)) = y;
    }
    wave_sync();
    if (LEAN) {   // (registers for keys or values at a time)
      __builtin_amdgcn_sched_barrier(0);
      load_keys();
    }
#pragma unroll
    for (int x = 0; x < 4 * KC; ++x) {
      f32x4& s = acc[0][0][x / (2 * KC)];
      const int y = x % (2 * KC);
      if (BF) {
        const uint4 qv = *reinterpret_cast<const uint4*>(qp + (y / 2) * 64 + (y % 2) * 8);
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kt[x]), __builtin_bit_cast(bf16x8, qv), s, 0, 0, 0);
      } else {
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, kt[x]), qf[y], s, 0, 0, 0);
      }
    }
    float p[1][1][8];
    weigh(acc, 1.4426950408889634f / sqrtf(static_cast<float>(HD)), 0.f, 1.f, false, tok0, true, p);
    union {
      uint16_t u[8];
      half8 h;
      bf16x8 b;
    } pf;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pf.u[e] = BF ? f2bf(p[0][0][e]) : f2h(p[0][0][e]);   // (rounded as the header of this part says)
      const int at = (e / 4) * 16 + g * 4 + e % 4;
      if (several && tok0 + at <= pos && bad[at]) l[0] = __uint_as_float(0x7FC00000u);   // (whatever it weighs: 0 times it is NaN)
    }
    // lane 4 a + b of a 16-lane group receives element b of the pieces that lanes a, a + 4, .. address
    lds_u16* const vl = (lds_u16*)(vt);
#pragma unroll
    for (int x = 0; x < NO; ++x) {
      v4i16 part[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int tok = tt * 16 + g * 4 + (c16 >> 2), d = x * 16 + 4 * (c16 & 3);
        part[tt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<lds_v4i16*>(vl + tok * HD + (((d >> 3) ^ (tok & 7)) << 3) + (d & 7)));
      }
      const auto vf = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
      o[0][x] = BF ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), pf.b, o[0][x], 0, 0, 0)
                   : __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, vf), pf.h, o[0][x], 0, 0, 0);
    }
  }
};

// floats of a state of `rows` rows in the waves alone: [rows][hd], [2][rows], a multiple of 4
static __host__ __device__ int alone_state(int rows, int hd) { return (rows * (hd + 2) + 3) / 4 * 4; }

// NW = 4: a workgroup per (tile, K/V head), or with SPLIT per segment of one.
// NW = 1: a wave per (tile, K/V head) takes the four shares of each segment one after another:
// the same sums, without the exchange.
template <int HD, bool BF, bool SPLIT, int NW>
__global__ __launch_bounds__(64 * NW, NW == 1 ? 3 : 2) void k_kv_attend(KvAttendArgs a, int64_t n_tiles, int32_t n_seg,
                                                                      int32_t slot_rows) {
  typedef KvWave<HD, BF, NW == 1> Wave;
  constexpr int NO = Wave::NO;
  __shared__ __attribute__((aligned(16))) uint16_t vt[KVB * HD];
  __shared__ int bad[KVB];
  extern __shared__ float lds[];
  float* so = lds;                               // NW = 4: [4][rows][HD]
  float* sm = so + (NW == 4 ? 4 * slot_rows * HD : 0);   // [4][rows]
  float* sl = sm + (NW == 4 ? 4 * slot_rows : 0);
  // of the earlier segments, where there are several: [rows][HD], [2][2][rows]; NW = 1: of the earlier shares
  // [rows][HD], [2][rows], then of the earlier segments the same (alone_state floats each, so that 16-byte accesses are aligned)
  float* state = sl + (NW == 4 ? 4 * slot_rows : 0);
  const KvCache& c = a.c;
  const int n = kv_count(a.b);
  if (n <= 0) return;
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rep = a.n_heads / c.n_kv;
  const int64_t tiles = a.b.cu ? unit_first(a.b, n, rep, 16, 1) : static_cast<int64_t>(n) * ((rep + 15) / 16);
  const int64_t items = (tiles < n_tiles ? tiles : n_tiles) * c.n_kv * (SPLIT ? n_seg : 1);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t unit = SPLIT ? item / n_seg : item;   // (tile, K/V head)
    const int seg0 = SPLIT ? static_cast<int>(item - unit * n_seg) : 0;
    const int64_t u = unit / c.n_kv;
    const int h = static_cast<int>(unit - u * c.n_kv);
    KvTile t;
    if (!kv_tile<16>(a, n, rep, u, t)) continue;
    const int segs = (t.nb + KV_SEG - 1) / KV_SEG;
    if (SPLIT && seg0 >= segs) continue;
    const int seg_end = SPLIT || segs == 0 ? seg0 + 1 : segs;
    Wave x(a, t, h, rep, vt, bad);
    if (NW == 1) {
      // states between shares and between segments: LDS (few rows; registers for them would cost a wave per SIMD)
      const int stride = alone_state(slot_rows, HD);
      auto fold = [&](bool any, const float* st) {   // the state st (none: !any), then this one, into (x.m, x.l, x.o)
        const bool is = any && c16 < t.rows;   // (a tile has slot_rows rows at most: a state holds no more)
        const float m0 = is ? st[slot_rows * HD + c16] : -INFINITY, l0 = is ? st[slot_rows * HD + slot_rows + c16] : 0.f;
        const float mn = fmaxf(m0, x.m[0]), ref = mn == -INFINITY ? 0.f : mn;
        const float e0 = __builtin_amdgcn_exp2f(m0 - ref), e1 = __builtin_amdgcn_exp2f(x.m[0] - ref);
        x.l[0] = fmaf(x.l[0], e1, l0 * e0);
#pragma unroll
        for (int y = 0; y < NO; ++y) {
          f32x4 z = f32x4{0.f, 0.f, 0.f, 0.f};
          if (is) z = *reinterpret_cast<const f32x4*>(st + c16 * HD + y * 16 + g * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.o[0][y][e] = fmaf(x.o[0][y][e], e1, z[e] * e0);
        }
        x.m[0] = mn;
      };
      auto keep = [&](float* st) {
        if (c16 < t.rows) {
#pragma unroll
          for (int y = 0; y < NO; ++y) *reinterpret_cast<f32x4*>(st + c16 * HD + y * 16 + g * 4) = x.o[0][y];
          if (g == 0) {
            st[slot_rows * HD + c16] = x.m[0];
            st[slot_rows * HD + slot_rows + c16] = x.l[0];
          }
        }
        wave_sync();
      };
      for (int seg = seg0; seg < seg_end; ++seg) {
        x.segment(seg);
        const int nbs = t.nb - seg * KV_SEG < KV_SEG ? t.nb - seg * KV_SEG : KV_SEG;
        const int full = x.full_blocks(seg, nbs);
        x.load(full > 0 ? 0 : -1);
        // share after share (blocks 0, 4, 8, 12, then 1, 5, ..), each folded onto those before
#pragma unroll 1
        for (int sh = 0; sh == 0 || (sh < 4 && sh < nbs); ++sh) {
          x.reset();
#pragma unroll 1
          for (int k = sh; k < full; k += 4)
            x.take(seg, k, k + 4 < full ? k + 4 : sh < 3 && sh + 1 < full ? sh + 1 : -1);
          if (full < nbs && (full & 3) == sh) x.tail((seg * KV_SEG + full) * KVB);
          x.l[0] = swap_add(x.l[0]);
          fold(sh > 0, state);
          if (sh < 3 && sh + 1 < nbs) keep(state);
        }
        fold(seg > seg0, state + stride);
        if (seg + 1 < seg_end) keep(state + stride);
      }
      if (c16 < t.rows) {
        const int q = t.r0 + c16;
        const float inv = kv_inverse(x.l[0], t.nb);
        uint16_t* op = a.out + (t.s.row0 + q / rep) * a.out_ld + (h * rep + q % rep) * HD + g * 4;
#pragma unroll
        for (int y = 0; y < NO; ++y) {
          uint32_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = f2act(x.o[0][y][e] * inv, a.out_act);
          *reinterpret_cast<uint2*>(op + y * 16) = make_uint2(v[0] | (v[1] << 16), v[2] | (v[3] << 16));
        }
      }
      wave_sync();
    } else {
      for (int seg = seg0; seg < seg_end; ++seg) {
        x.segment(seg);
        const int nbs = t.nb - seg * KV_SEG < KV_SEG ? t.nb - seg * KV_SEG : KV_SEG;
        x.reset();
        const int full = x.full_blocks(seg, nbs);
        x.load(w < full ? w : -1);
#pragma unroll 1
        for (int k = w; k < full; k += 4) x.take(seg, k, k + 4 < full ? k + 4 : -1);
        if (full < nbs && (full & 3) == w) x.tail((seg * KV_SEG + full) * KVB);
        const float lw = swap_add(x.l[0]);
        __syncthreads();   // the last segment's states are read before these are written
        if (c16 < t.rows) {
#pragma unroll
          for (int y = 0; y < NO; ++y)
            *reinterpret_cast<f32x4*>(so + (w * slot_rows + c16) * HD + y * 16 + g * 4) = x.o[0][y];
          if (g == 0) {
            sm[w * slot_rows + c16] = x.m[0];
            sl[w * slot_rows + c16] = lw;
          }
        }
        __syncthreads();
        // the shares folded in order, then onto the earlier segments' state (its sums by parity)
#pragma unroll 1
        for (int e = threadIdx.x; e < t.rows * HD; e += 64 * NW) {
          const int r = e / HD, d = e % HD;
          float m1 = -INFINITY, l1 = 0.f, o1 = 0.f;
#pragma unroll
          for (int v = 0; v < 4; ++v)
            kv_fold(m1, l1, o1, sm[v * slot_rows + r], sl[v * slot_rows + r], so[(v * slot_rows + r) * HD + d]);
          float m0 = -INFINITY, l0 = 0.f, o0 = 0.f;
          if (!SPLIT && seg > 0) {
            const float* st = state + slot_rows * HD + (seg & 1) * 2 * slot_rows;
            m0 = st[r];
            l0 = st[slot_rows + r];
            o0 = state[e];
          }
          kv_fold(m0, l0, o0, m1, l1, o1);
          if (!SPLIT && seg + 1 < seg_end) {
            float* st = state + slot_rows * HD + ((seg + 1) & 1) * 2 * slot_rows;
            state[e] = o0;
            if (d == 0) {
              st[r] = m0;
              st[slot_rows + r] = l0;
            }
          } else if (SPLIT) {   // the segment's state: values, then (reference, sum) per row
            float* slot = a.part + (unit * n_seg + seg0) * (static_cast<int64_t>(slot_rows) * (HD + 2));
            slot[e] = o0;
            if (d == 0) {
              slot[slot_rows * HD + 2 * r] = m0;
              slot[slot_rows * HD + 2 * r + 1] = l0;
            }
          } else {
            const int q = t.r0 + r;
            const float v = o0 * kv_inverse(l0, t.nb);
            a.out[(t.s.row0 + q / rep) * a.out_ld + (h * rep + q % rep) * HD + d] = f2act(v, a.out_act);
          }
        }
      }
      __syncthreads();
    }
  }
}

// Folds the segments' states of each tile, in order, JOIN segments at a time: a wave per row finds how its reference
// rises (a scan over the segments, a lane each) and the fold's factors, then every thread takes its values'
// chain of multiply-adds with the first 32 segments' values read ahead.  Bound by the latency of those reads: 23 us for
// 196 segments of 32 tiles (6.4 MB); with the chain of maxima and exponentials in every thread it took 70.
constexpr int JOIN = 64;
template <int HD>
__global__ __launch_bounds__(256) void k_kv_join(KvAttendArgs a, int64_t n_tiles, int32_t n_seg, int32_t slot_rows) {
  __shared__ float fx[JOIN][16], fy[JOIN][16], fl[JOIN][16], top[16], sum[16];
  const KvCache& c = a.c;
  const int n = kv_count(a.b);
  if (n <= 0) return;
  const int rep = a.n_heads / c.n_kv;
  const int64_t unit = blockIdx.x;
  const int64_t u = unit / c.n_kv;
  const int h = static_cast<int>(unit - u * c.n_kv);
  const int64_t tiles = a.b.cu ? unit_first(a.b, n, rep, 16, 1) : static_cast<int64_t>(n) * ((rep + 15) / 16);
  if (u >= tiles || u >= n_tiles) return;
  KvTile t;
  if (!kv_tile<16>(a, n, rep, u, t)) return;
  const int segs = (t.nb + KV_SEG - 1) / KV_SEG;
  const int64_t step = static_cast<int64_t>(slot_rows) * (HD + 2);
  const float* slot = a.part + unit * n_seg * step;
  constexpr int PER = 16 * HD / 256;
  const int used = (t.rows * HD + 255) / 256;   // values of a thread
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  float o[PER], l = 0.f;
#pragma unroll
  for (int x = 0; x < PER; ++x) o[x] = 0.f;
  if (threadIdx.x < 16) top[threadIdx.x] = -INFINITY;
  for (int s0 = 0; s0 < segs; s0 += JOIN) {
    const int ns = segs - s0 < JOIN ? segs - s0 : JOIN;
    float v[32];
    auto read = [&](int x, int s) {   // the segments' values from s on
      const int e = threadIdx.x + x * 256;
      const float* p = slot + s0 * step + (e < t.rows * HD ? e : 0);
#pragma unroll
      for (int q = 0; q < 32; ++q) v[q] = p[(s + q < ns ? s + q : ns - 1) * step];
    };
    read(0, 0);
    __syncthreads();
    for (int r = w; r < t.rows; r += 4) {   // a wave per row, a lane per segment: the references as they rise, kv_fold's factors
      const float* ml = slot + (s0 + (lane < ns ? lane : 0)) * step + slot_rows * HD + 2 * r;
      const float mp = lane < ns ? ml[0] : -INFINITY, lp = ml[1], first = top[r];
      float m = mp;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const float y = __shfl_up(m, d);
        m = lane >= d ? fmaxf(m, y) : m;
      }
      m = fmaxf(m, first);
      const float up = __shfl_up(m, 1), before = lane ? up : first, ref = m == -INFINITY ? 0.f : m;
      fx[lane][r] = __builtin_amdgcn_exp2f(before - ref);
      fy[lane][r] = __builtin_amdgcn_exp2f(mp - ref);
      fl[lane][r] = lp;
      if (lane == 63) top[r] = m;
    }
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < t.rows) {
      const int r = threadIdx.x;
#pragma unroll 8
      for (int s = 0; s < ns; ++s) l = fmaf(fl[s][r], fy[s][r], l * fx[s][r]);
      sum[r] = l;
    }
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      if (x >= used) break;
      const int e = threadIdx.x + x * 256, r = e / HD < t.rows ? e / HD : 0;
      for (int s = 0; s < ns; s += 32) {
        if (x > 0 || s > 0) read(x, s);
#pragma unroll
        for (int q = 0; q < 32; ++q)
          if (s + q < ns) o[x] = fmaf(v[q], fy[s + q][r], o[x] * fx[s + q][r]);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int e = threadIdx.x + x * 256;
    if (e >= t.rows * HD) break;
    const int r = e / HD, d = e % HD, q = t.r0 + r;
    const float v = segs == 0 ? 0.f : o[x] * kv_inverse(sum[r], t.nb);
    a.out[(t.s.row0 + q / rep) * a.out_ld + (h * rep + q % rep) * HD + d] = f2act(v, a.out_act);
  }
}

// ------------------------------------------------------------------ several rows per sequence
// A workgroup of four waves per 128 query rows of a (sequence, K/V head), 32 rows
// (two lane-column tiles) per wave, all waves walking the same blocks, two at a step: a block's bytes
// become fp16 fragments once per workgroup, in LDS, in the order in which the products
// take them (every access 16 bytes per lane, in lane order), the next two steps' bytes in
// flight meanwhile.  Bound: the softmax's VALU work (16 scores per lane and block of
// 32 keys, 8 exponentials of 4 issue slots each per tile) and 32 matrix instructions, by turns: two waves per SIMD overlap
// little of them.  64 sequences of about 900 tokens with 128 new ones, 24/8 heads of 128: 155 us, 650
// TFLOP/s of products that are seen, CUs busy 86% of the time, vector instructions in issue 45%, matrix units busy
// 28%, LDS busy 25% (a fragment read feeds two products; no bank conflicts) and 3% of the waves' time spent waiting to issue
// to it; 16 sequences of 4,000 with 512 830 TFLOP/s.
constexpr int KV_ROWS = 128;
constexpr int KV_LIST = 64;      // numbers and scales of twice as many blocks are in LDS
constexpr int KV_AHEAD = 4;      // blocks whose bytes are in flight or staged

// The tiles of a batch of up to 256 sequences in the order of descending lengths, so that long ones do not start last:
// lengths by class, sixteen to an octave below max_len, sequences of a class in their own order.
struct KvOrder {
  int tiles[128];            // of the classes
  int sum[4], first;
  KvRaw seq;
};
// a value's sum over the lanes up to each (row_shr 1, 2, 4, 8, row_bcast 15, 31)
__device__ __forceinline__ int lanes_upto(int v) {
#define AIQ_STEP(CTRL_, ROWS_) v += __builtin_amdgcn_update_dpp(0, v, CTRL_, ROWS_, 0xF, false)
  AIQ_STEP(0x111, 0xF);
  AIQ_STEP(0x112, 0xF);
  AIQ_STEP(0x114, 0xF);
  AIQ_STEP(0x118, 0xF);
  AIQ_STEP(0x142, 0xA);
  AIQ_STEP(0x143, 0xC);
#undef AIQ_STEP
  return v;
}
// Tile u: its sequence and the first tile of that; false: past the last.  All threads together.
__device__ __forceinline__ bool kv_order(const KvAttendArgs& a, int n, int rep, int R, int64_t u, KvOrder& s, KvRaw& seq, int& first) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  KvRaw raw;   // this thread's sequence, its tiles, its class
  int tiles = 0, cls = 127;
  if (tid < n) {
    const KvAt q{a.b, tid};
    raw = {{q.len(), q.c0(), q.c1(), q.e0(), q.e1(), q.tail()}};
  }
  if (tid < 128) s.tiles[tid] = 0;
  if (tid < n) {
    const int64_t rows = static_cast<int64_t>(raw.c1()) - raw.c0();
    tiles = rows < 0 || rows > a.b.n_rows ? 1 : static_cast<int>((rows * rep + R - 1) / R);   // (1: to be flagged)
    auto log16 = [](int x) { return static_cast<int>(__float_as_uint(static_cast<float>(x < 1 ? 1 : x)) >> 19); };
    const int below = log16(a.b.max_len) - log16(raw.len());
    cls = below < 0 ? 0 : below > 127 ? 127 : below;
  }
  __syncthreads();
  if (tiles > 0) atomicAdd(&s.tiles[cls], tiles);
  __syncthreads();
  const int t0 = s.tiles[2 * lane], t1 = s.tiles[2 * lane + 1], upto = lanes_upto(t0 + t1), before = upto - t0 - t1;
  const uint64_t hit = __ballot(before <= u && u < upto);
  if (!hit) return false;
  const int at = __builtin_ctzll(hit);
  const int b0 = __builtin_amdgcn_readlane(before, at), f0 = __builtin_amdgcn_readlane(t0, at);
  const bool second = u - b0 >= f0;
  const int c = 2 * at + second, mine = cls == c ? tiles : 0, in = lanes_upto(mine);
  if (lane == 63) s.sum[w] = in;
  __syncthreads();
  int from = b0 + (second ? f0 : 0) + in - mine;
  for (int x = 0; x < w; ++x) from += s.sum[x];
  if (mine > 0 && from <= u && u < from + mine) {
    s.seq = raw;
    s.first = from;
  }
  __syncthreads();
  seq = s.seq;
  first = uniform(s.first);
  return true;
}

template <int HD, bool BF, bool ORDER>
__global__ __launch_bounds__(256, HD == 64 ? 3 : 2) void k_kv_attend_rows(KvAttendArgs a, int64_t n_tiles) {
  constexpr int KC = HD / 64, NO = HD / 16, FR = 2 * KC;   // FR fragments of 16 bytes per lane of keys, and of values
  constexpr int PER = 2 * FR * 64 / 256;                   // of them per thread
  // [buffer][block][keys, values][fragment][half][lane] of 8 fp16 (the tail of a bf16 cache: bf16)
  __shared__ __attribute__((aligned(16))) uint16_t frag[2][2][2][FR][2][64][8];
  __shared__ int ids[2 * KV_LIST];
  __shared__ KvScale scales[2 * KV_LIST];
  __shared__ int bad[KVB];
  const KvCache& c = a.c;
  const int n = kv_count(a.b);
  if (n <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rep = a.n_heads / c.n_kv;
  __shared__ std::conditional_t<ORDER, KvOrder, int> ord;
  int64_t items = n_tiles * c.n_kv;
  if constexpr (!ORDER) {
    const int64_t tiles = unit_first(a.b, n, rep, KV_ROWS, 1);
    if (tiles < n_tiles) items = tiles * c.n_kv;
  }
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t u = item / c.n_kv;
    const int h = static_cast<int>(item - u * c.n_kv);
    KvTile t;
    if constexpr (ORDER) {
      KvRaw raw;
      int first;
      if (!kv_order(a, n, rep, KV_ROWS, u, ord, raw, first) || !kv_tile<KV_ROWS>(a, n, rep, u - first, t, &raw)) return;
    } else if (!kv_tile<KV_ROWS>(a, n, rep, u, t)) {
      continue;
    }
    const int base = t.s.len - t.s.n;
    // queries of tile x: row w * 32 + x * 16 + c16
    const uint16_t* qp[2];
    half8 qf[2][FR];
    float fac[2], m[2], l[2];
    int pos[2];
    f32x4 o[2][NO];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = w * 32 + x * 16 + c16, row = t.r0 + (r < t.rows ? r : t.rows - 1);
      pos[x] = base + row / rep;
      qp[x] = a.q + (t.s.row0 + row / rep) * a.q_ld + (h * rep + row % rep) * HD + g * 16;
#pragma unroll
      for (int y = 0; y < FR; ++y) qf[x][y] = __builtin_bit_cast(half8, *reinterpret_cast<const uint4*>(qp[x] + (y / 2) * 64 + (y % 2) * 8));
      fac[x] = 1.4426950408889634f / sqrtf(static_cast<float>(HD));
      if (BF) fac[x] *= rows_f16<FR>(qf[x]);
      m[x] = -INFINITY;
      l[x] = 0.f;
#pragma unroll
      for (int y = 0; y < NO; ++y) o[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // positions of the wave's first and last row: blocks past the last are not its, up to the first all of it is seen
    const int wr = w * 32 < t.rows ? w * 32 : t.rows - 1, we = w * 32 + 31 < t.rows ? w * 32 + 31 : t.rows - 1;
    const int first = base + (t.r0 + wr) / rep, last = w * 32 < t.rows ? base + (t.r0 + we) / rep : -1;
    const int full = t.s.len / KVB < t.nb ? t.s.len / KVB : t.nb;   // the tile's blocks that are not the tail
    uint4 even[2][PER], odd[2][PER];   // bytes of the blocks of even pairs, of odd ones
    auto list = [&](int j0) {   // blocks j0 .. j0 + KV_LIST - 1, in the half of the list whose blocks are long past
      if (tid < KV_LIST) {
        const int to = (j0 + tid) % (2 * KV_LIST), id = j0 + tid < full ? kv_block(c, a.b, t.s.bs + j0 + tid) : -1;
        ids[to] = id < 0 ? 0 : id;
        const int64_t at = static_cast<int64_t>(id) * c.n_kv + h;
        scales[to] = id < 0 ? KvScale{1.f, -INFINITY, 1.f, false} : kv_scale(c.ks[at], c.vs[at]);
      }
      __syncthreads();
    };
    auto load = [&](uint4 (&r)[PER], int j) {
      if (j >= full) return;
      const int64_t at = (static_cast<int64_t>(uniform(ids[j % (2 * KV_LIST)])) * c.n_kv + h) * (KVB * HD);
#pragma unroll
      for (int x = 0; x < PER; ++x) {   // fragment (x * 4 + w), keys first
        const int f = x * 4 + w;
        r[x] = *reinterpret_cast<const uint4*>((f < FR ? c.k + at + f * 1024 : c.v + at + (f - FR) * 1024) +
                                               static_cast<uint32_t>(lane) * 16);
      }
    };
    auto stage = [&](const uint4 (&r)[PER], int buf, int s) {
#pragma unroll
      for (int x = 0; x < PER; ++x) {
        const int f = x * 4 + w;
        *reinterpret_cast<half8*>(frag[buf][s][f / FR][f % FR][0][lane]) = bytes_f16(r[x].x, r[x].y);
        *reinterpret_cast<half8*>(frag[buf][s][f / FR][f % FR][1][lane]) = bytes_f16(r[x].z, r[x].w);
      }
    };
    list(0);
#pragma unroll
    for (int d = 0; d < 2; ++d) {
#pragma unroll
      for (int x = 0; x < PER; ++x) even[d][x] = odd[d][x] = make_uint4(0, 0, 0, 0);   // (a pair's second block where there is none: weighs nothing)
      load(even[d], d);
      load(odd[d], 2 + d);
    }
    stage(even[0], 0, 0);
    stage(even[1], 0, 1);
    // blocks j and j + 1, staged in buf; the next pair's bytes are in `next`, those of the pair after it go into `then`
    auto step = [&](int j, int buf, const uint4 (&next)[2][PER], uint4 (&then)[2][PER]) {
      const KvScale sc[2] = {scales[j % (2 * KV_LIST)], scales[(j + 1) % (2 * KV_LIST)]};
      if ((j + KV_AHEAD) % KV_LIST == 0) list(j + KV_AHEAD);
      load(then[0], j + KV_AHEAD);
      load(then[1], j + KV_AHEAD + 1);
      __syncthreads();   // blocks j, j + 1 staged; the other buffer's consumed
      const int tok0 = j * KVB;
      if (tok0 <= last) {
        f32x4 acc[2][2][2];
        float c1[2][2], p[2][2][8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            acc[s][x][0] = acc[s][x][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            c1[s][x] = kv_factor(fac[x], sc[s].k);
          }
#pragma unroll
          for (int f = 0; f < FR; ++f)   // tile f / KC of 16 tokens, 64-dim slice f % KC
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const half8 kf = *reinterpret_cast<const half8*>(frag[buf][s][0][f][e][lane]);
#pragma unroll
              for (int x = 0; x < 2; ++x)
                acc[s][x][f / KC] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[x][(f % KC) * 2 + e], acc[s][x][f / KC], 0, 0, 0);
            }
        }
        const bool masked = tok0 + 2 * KVB - 1 > first;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int x = 0; x < 2; ++x) kv_mask(acc[s][x], uniform(sc[s].bad) != 0, masked, tok0 + s * KVB + g * 4, pos[x]);
        const float c2[2] = {sc[0].log_v, sc[1].log_v}, inv[2] = {sc[0].inv_v, sc[1].inv_v};
        kv_softmax<2, 2, NO>(acc, c1, c2, inv, m, l, o, p);
        half8 pf[2][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[s][x][e] = static_cast<_Float16>(p[s][x][e]);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int f = 0; f < FR; ++f)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const half8 vf = *reinterpret_cast<const half8*>(frag[buf][s][1][f][e][lane]);
#pragma unroll
              for (int x = 0; x < 2; ++x) o[x][2 * f + e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[s][x], o[x][2 * f + e], 0, 0, 0);
            }
      }
      if (j + 2 < full) {
        stage(next[0], buf ^ 1, 0);
        stage(next[1], buf ^ 1, 1);
      }
    };
    for (int j = 0; j < full; j += 4) {
      step(j, 0, odd, even);
      if (j + 2 < full) step(j + 2, 1, even, odd);
    }
    if (full < t.nb) {   // the tail: its rows as fragments of their own type
      const int tok0 = full * KVB, left = t.s.len - tok0;
      const uint16_t* tk = tail_at(c, t.s.tail, 0, h);
      const uint16_t* tv = tail_at(c, t.s.tail, 1, h);
      __syncthreads();
      if (tid < KVB) bad[tid] = 0;
      __syncthreads();
      for (int x = tid; x < FR * 2 * 64; x += 256) {
        const int f = x / 128, e = x / 64 % 2, ln = x % 64, gg = ln >> 4, cc = ln & 15;
        const int tok = (f / KC) * 16 + cc, row = tok < left ? tok : left - 1;
        *reinterpret_cast<uint4*>(frag[0][0][0][f][e][ln]) =
            *reinterpret_cast<const uint4*>(tk + static_cast<uint32_t>(row * HD + (f % KC) * 64 + gg * 16 + e * 8));
        union {
          uint16_t u[8];
          uint4 q;
        } v;
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int vt = (y / 4) * 16 + gg * 4 + y % 4, vr = vt < left ? vt : left - 1;
          v.u[y] = tv[static_cast<uint32_t>(vr * HD + f * 32 + e * 16 + cc)];
        }
#pragma unroll
        for (int y = 0; y < 8; ++y) {   // a later query's infinity or NaN must not meet the weight 0
          const int vt = (y / 4) * 16 + gg * 4 + y % 4;
          const bool inf = (v.u[y] & 0x7FFFu) >= (BF ? 0x7F80u : 0x7C00u);
          if (inf && vt < left) bad[vt] = 1;
          if (inf || vt >= left) v.u[y] = 0;
        }
        *reinterpret_cast<uint4*>(frag[0][0][1][f][e][ln]) = v.q;
      }
      __syncthreads();
      if (tok0 <= last) {
        f32x4 acc[1][2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          acc[0][x][0] = acc[0][x][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int f = 0; f < FR; ++f)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint4 kf = *reinterpret_cast<const uint4*>(frag[0][0][0][f][e][lane]);
              const int y = (f % KC) * 2 + e;
              f32x4& s = acc[0][x][f / KC];
              if (BF) {
                const uint4 qv = *reinterpret_cast<const uint4*>(qp[x] + (y / 2) * 64 + (y % 2) * 8);
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qv), s, 0, 0, 0);
              } else {
                s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, kf), qf[x][y], s, 0, 0, 0);
              }
            }
        }
        float p[1][2][8];
        const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(HD)), c1[1][2] = {{scale, scale}}, none[1] = {0.f}, one[1] = {1.f};
#pragma unroll
        for (int x = 0; x < 2; ++x) kv_mask(acc[0][x], false, true, tok0 + g * 4, pos[x]);
        kv_softmax<1, 2, NO>(acc, c1, none, one, m, l, o, p);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          union {
            uint16_t u[8];
            half8 h;
            bf16x8 b;
          } pf;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            pf.u[e] = BF ? f2bf(p[0][x][e]) : f2h(p[0][x][e]);
            const int at = (e / 4) * 16 + g * 4 + e % 4;
            if (tok0 + at <= pos[x] && bad[at]) l[x] = __uint_as_float(0x7FC00000u);   // (whatever it weighs: 0 times it is NaN)
          }
#pragma unroll
          for (int f = 0; f < FR; ++f)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint4 vf = *reinterpret_cast<const uint4*>(frag[0][0][1][f][e][lane]);
              o[x][2 * f + e] = BF ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), pf.b, o[x][2 * f + e], 0, 0, 0)
                                   : __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, vf), pf.h, o[x][2 * f + e], 0, 0, 0);
            }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = w * 32 + x * 16 + c16;
      const float lw = swap_add(l[x]), inv = kv_inverse(lw, t.nb);
      if (r < t.rows) {
        const int q = t.r0 + r;
        uint16_t* op = a.out + (t.s.row0 + q / rep) * a.out_ld + (h * rep + q % rep) * HD + g * 4;
#pragma unroll
        for (int y = 0; y < NO; ++y) {
          uint32_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = f2act(o[x][y][e] * inv, a.out_act);
          *reinterpret_cast<uint2*>(op + y * 16) = make_uint2(v[0] | (v[1] << 16), v[2] | (v[3] << 16));
        }
      }
    }
    if (ORDER) return;   // (a workgroup per item)
    __syncthreads();
  }
}

struct KvShape {
  int64_t tiles;     // bound on the batch's tiles
  int32_t n_seg;     // segments of the longest sequence
  int32_t rows;      // rows of a tile that can be in use
  bool split, alone;
  bool many;         // many rows per sequence: tiles of KV_ROWS
};
static KvShape kv_shape(const KvCache& c, const KvBatch& b, int32_t n_heads) {
  const int rep = n_heads / c.n_kv;
  KvShape s{};
  s.tiles = b.cu ? b.n_rows * rep / 16 + b.n_seq : static_cast<int64_t>(b.n_seq) * ((rep + 15) / 16);
  s.n_seg = (b.max_len + KV_SEG * KVB - 1) / (KV_SEG * KVB);
  s.rows = b.cu || rep > 16 ? 16 : rep;
  const int64_t big = b.cu ? b.n_rows * rep / KV_ROWS + b.n_seq : 0;
  // Tiles of KV_ROWS rows against tiles of 16, 24/8 heads of 128 and 32/8 heads of 64: 256 sequences of about 300 tokens
  // with 8 new rows each 81 us against 71 and 45 against 38, with 16 (48 and 64 rows per K/V head) 90 against 124
  // and 54 against 58, with 32 101 against 191 and 58 against 97; 64 sequences of 900 with 16 48 against 95 and 35
  // against 56.  Where the tiles of 16 are few they run at once, four waves to a tile's keys: 16 sequences of 2,000 with
  // 16 (512 and 640 of them) 65 against 47 and 48 against 37, with 32 (896, 1,152) 67 against 81 and 52 against 57; 4 of
  // 4,000 with 64 (416, 544) 116 against 83 and 84 against 64, with 128 (800, 1,056) 121 against 137 and 87 against 93.
  // (Between one row and those: 8 new rows of three heads are two tiles of 16, each reading all of the sequence's bytes, 66 us
  // where the bytes take 38.)
  // (One row per sequence stays with the tiles of 16 whatever its heads: their order of sums is the keys' alone.)
  s.many = b.cu && b.n_rows > b.n_seq && b.n_rows * rep >= static_cast<int64_t>(b.n_seq) * KV_MANY &&
           s.tiles * c.n_kv >= 768;
  if (s.many) {
    s.tiles = big;
    return s;
  }
  // Inside a query n_seq is the most sequences that a pass may hold, not how many the query selects (n_ptr): a selective
  // one takes the rules' side for many.
  const int64_t items = s.tiles * c.n_kv;
  // Segments in workgroups of their own where (tile, K/V head) items leave CUs without work for long enough
  // to pay for the second launch (about 5 us).  Split against one workgroup per item, heads of 64: 8 items of
  // 800, 1,500 and 4,000 tokens 9.8, 10.4 and 10.4 us against 8.2, 11.6 and 25.4; 64 items of 1,500 10.8 against
  // 11.8; 256 items of 1,500 and 4,000 18.1 and 29.2 against 16.0 and 34.3 (24/8 heads of 128: 30 and 54
  // against 23 and 48); 512 items of 4,000 48 against 45.  Among more items only very long
  // sequences, which a ragged batch may have one of.
  s.split = !b.n_ptr && ((s.n_seg >= 3 && items < 256) || (s.n_seg >= 16 && items < 1024));
  // Waves alone where the items fill the chip and none of them is a long chain for its wave.  Alone against a
  // workgroup per item, heads of 64: 2,048 items of 150 (up to 750) tokens 25.4 us against 19.4, 4,096 32.1 against
  // 30.3, 8,192 46.8 against 54.2; 2,048 of 30 9.8 against 11.7, of 600 (up to 3,000) 72 against 46; heads of
  // 128 (groups of 3): 2,048 of 150 34.2 against 35.4, 4,096 48 against 62, 2,048 of 600 139 against 100.
  s.alone = !s.split && items >= 2048 && items >= static_cast<int64_t>(b.max_len) * (c.hd == 64 ? 6 : 3);
  return s;
}

size_t kv_attend_part_bytes(const KvCache& c, const KvBatch& b, int32_t n_heads) {
  const KvShape s = kv_shape(c, b, n_heads);
  if (!s.split) return 0;
  return static_cast<size_t>(s.tiles) * c.n_kv * s.n_seg * s.rows * (c.hd + 2) * 4;
}

hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t s) {
  if (a.b.n_seq == 0 || a.b.n_rows == 0) return hipSuccess;
  if (a.c.hd != 64 && a.c.hd != 128) return hipErrorInvalidValue;
  const KvShape k = kv_shape(a.c, a.b, a.n_heads);
  if (k.split && !a.part) return hipErrorInvalidValue;
  const int64_t items = k.tiles * a.c.n_kv * (k.split ? k.n_seg : 1);
  const bool bf = a.c.act == ACT_BF16;
  if (k.many) {
    const dim3 grid(static_cast<unsigned>(items < (1 << 20) ? items : 1 << 20));
    // In the order of lengths, without empty tiles, against the order of the batch (a tile more per sequence than its rows
    // may need), 24/8 heads of 128 and 32/8 heads of 64: 64 sequences of about 900 tokens (sigma 0.4) with 128 new rows
    // 160 us against 220 and 118 against 139; 256 of 300 with 32 116 against 143 and 61 against 119; 256 of 40 with
    // 256 411 against 402 and 314 against 298.
    const bool order = a.b.n_seq <= 256 && items <= 1 << 20;   // (a thread per sequence, a workgroup per tile)
#define AIQ_KV_ROWS(HD_, BF_)                                                                            \
  if (order) hipLaunchKernelGGL((k_kv_attend_rows<HD_, BF_, true>), grid, dim3(256), 0, s, a, k.tiles);  \
  else hipLaunchKernelGGL((k_kv_attend_rows<HD_, BF_, false>), grid, dim3(256), 0, s, a, k.tiles)
    if (a.c.hd == 64 && bf) {
      AIQ_KV_ROWS(64, true);
    } else if (a.c.hd == 64) {
      AIQ_KV_ROWS(64, false);
    } else if (bf) {
      AIQ_KV_ROWS(128, true);
    } else {
      AIQ_KV_ROWS(128, false);
    }
#undef AIQ_KV_ROWS
    return hipGetLastError();
  }
  const int64_t cap = !a.b.n_ptr ? 1 << 20 : k.alone ? 1 << 16 : 1 << 14;   // (a bound from the host only: the sequences may be few)
  const dim3 grid(static_cast<unsigned>(items < cap ? items : cap));
  const int state = 4 * (a.c.hd + 2) + (!k.split && k.n_seg > 1 ? a.c.hd + 4 : 0);   // per row, of four waves
  const size_t lds = static_cast<size_t>(k.alone ? 2 * alone_state(k.rows, a.c.hd) : k.rows * state) * 4;
#define AIQ_KV_ATTEND(HD_, BF_, SP_, NW_) \
  hipLaunchKernelGGL((k_kv_attend<HD_, BF_, SP_, NW_>), grid, dim3(64 * NW_), lds, s, a, k.tiles, k.n_seg, k.rows)
#define AIQ_KV_ATTEND_BF(HD_, BF_)                       \
  if (k.split) AIQ_KV_ATTEND(HD_, BF_, true, 4);         \
  else if (k.alone) AIQ_KV_ATTEND(HD_, BF_, false, 1);     \
  else AIQ_KV_ATTEND(HD_, BF_, false, 4)
  if (a.c.hd == 64 && bf) {
    AIQ_KV_ATTEND_BF(64, true);
  } else if (a.c.hd == 64) {
    AIQ_KV_ATTEND_BF(64, false);
  } else if (a.c.hd == 128 && bf) {
    AIQ_KV_ATTEND_BF(128, true);
  } else if (a.c.hd == 128) {
    AIQ_KV_ATTEND_BF(128, false);
  } else {
    return hipErrorInvalidValue;
  }
#undef AIQ_KV_ATTEND_BF
#undef AIQ_KV_ATTEND
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !k.split) return e;
  const dim3 jg(static_cast<unsigned>(k.tiles * a.c.n_kv));
  if (a.c.hd == 64)
    hipLaunchKernelGGL((k_kv_join<64>), jg, dim3(256), 0, s, a, k.tiles, k.n_seg, k.rows);
  else
    hipLaunchKernelGGL((k_kv_join<128>), jg, dim3(256), 0, s, a, k.tiles, k.n_seg, k.rows);
  return hipGetLastError();
}

}  // namespace aiq
