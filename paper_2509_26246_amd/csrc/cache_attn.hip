// Attention of each sequence's last rows over its 4-bit cache (layout: cache.h), few rows per sequence: single tokens, drafted tokens.
//
// Mathematics.  S = K q over the codes: the 32 channels of a scale group are one 16x16x32 product, whose 16 keys x 16 query columns are then
// multiplied by the keys' scales in fp32 and added up over the groups: no value of K is ever formed, and q enters as it is.  Likewise
// O^T = V^T P^T takes V's codes as they are, and the probabilities of a scale group times that group's scales (rounded to bf16 as P would
// be).  fp32 calls hand q and P over as three bf16 terms, 24 bits: with exact codes the products are then as good as fp32 ones.
// Softmax statistics and sums are fp32, in log2 units; the maximum moves with every step.
//
// Bound by memory (144 bytes per key and KV head at head dim 128 against 4 * 128 flops per query head), so what counts is that every compute unit reads
// all the time, whatever the lengths are.  The columns of a sequence's KV head (rows x heads of the group) are cut into tiles of 16, an item is
// one tile's walk over the keys it sees, its length counted in units of 256 keys; the units of all items in a row are divided evenly among
// the blocks of one launch, which find their place in that row by a scan over the lengths (they are data: a recorded call follows
// them).  A block's first and last item may be parts; parts leave O, maximum and sum in the workspace, and a second launch adds them up in the
// order of the keys.  A unit is 4 waves x 64 keys; each wave keeps its own state and shares nothing before the end of an item.
//
// A wave's step, 64 keys (lane group h = lane / 16 holds keys 16h .. 16h+15 of everything): the next step's codes and scales are loaded while
// this one is computed; K codes go from the load to the conversion (the cache holds them in operand order), V codes and all scales
// through the wave's own LDS, where the 4-bit transpose read turns rows of V into the operand's columns.
#include <hip/hip_runtime.h>

#include "cache.h"

namespace slimattn {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kCols = 16;            // query columns of a tile
constexpr int kStep = 64;            // keys of a wave's step
constexpr int kUnit = kWaves * kStep;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxGrid = 1024;       // four blocks per compute unit

struct AttnArgs {
  CacheView c;
  int group, Hq;                     // query heads per KV head; of all
  float scale_log2;                  // > 0
  float q_sign;                      // scale < 0 turns q around; 0 makes it zero
};

// A split item, written by the block that holds its start, for the launch that adds its parts up.
struct Split { int first, parts, row0, cols, col0, head0; };
struct Header { int blocks, pad[7]; };

template <int D> constexpr int kPartFloats = kCols * D + 2 * kCols;   // [col][D], max [col], sum [col]

template <int D>
__device__ __forceinline__ float* part_of(char* ws, int block, int slot) {
  return reinterpret_cast<float*>(ws + sizeof(Header) + (size_t)kMaxGrid * 32) + ((size_t)block * 2 + slot) * kPartFloats<D>;
}

typedef float floatx4v __attribute__((ext_vector_type(4)));
typedef int int2v __attribute__((ext_vector_type(2)));
template <int D> struct Piece;                    // what a lane loads of D/2 bytes x 16 keys, or of the scales
template <> struct Piece<128> { typedef uint4 type; };
template <> struct Piece<64> { typedef uint2 type; };

__device__ __forceinline__ unsigned word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ unsigned word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

__device__ __forceinline__ floatx4v mfma16(bf16x8 a, bf16x8 b, floatx4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// x as a sum of TERMS bf16 values, the largest first (each takes eight bits of what is left).
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8 (&t)[TERMS]) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int n = 0; n < TERMS; ++n)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[n][i] = (bf16)rest[i];
      rest[i] -= (float)t[n][i];
    }
}

// LDS of one wave: V codes (rows of D/2 bytes, 16 more to spread the transpose reads over the banks), K scales, V scales.
template <int D> constexpr int kVRow = D / 2 + 16;
template <int D> constexpr int kScaleBytes = kStep * (D / 16);
template <int D> constexpr int kWaveLds = kStep * kVRow<D> + 2 * kScaleBytes<D>;
template <int D> constexpr int kOutRow = D + 4;                                    // floats; at the end: [wave][col][kOutRow], max, sum
template <int D> constexpr int kEndLds = kWaves * kCols * (kOutRow<D> + 2) * 4;
template <int D> constexpr int kLds = kWaves * kWaveLds<D> > kEndLds<D> ? kWaves * kWaveLds<D> : kEndLds<D>;

// One step's loads.
template <int D>
struct StepData {
  typedef typename Piece<D>::type P;
  P k[4], v[4], s;
  unsigned ok;                       // bit h: the keys 16h .. 16h+15 are in a page (uniform)
};

template <int D>
__device__ __forceinline__ void load_step(StepData<D>& x, const CacheView& c, const char* cache, int b, int hk, int k0, int visible) {
  typedef typename Piece<D>::type P;
  const int lane = threadIdx.x & 63, P_mask = (1 << c.page_shift) - 1;
  const int chunk = (lane >> 2) & 3, key = k0 + kCacheChunk * chunk;
  int page = key < visible ? page_at(c, b, key) : -1;
  const unsigned long long good = __ballot(page >= 0);
  x.ok = (unsigned)(good & 1) | (unsigned)((good >> 4 & 1) << 1) | (unsigned)((good >> 8 & 1) << 2) | (unsigned)((good >> 12 & 1) << 3);
  page = max(page, 0);               // chunks without a page read page 0 and are masked
  const long long piece = hk * head_bytes<D>(c), pb = page_bytes<D>(c);
  const char* kp = cache + page * pb + piece + key_codes<D>((key & P_mask) + (lane & 3)) + (lane >> 4) * (D / 8);
#pragma unroll
  for (int t = 0; t < 4; ++t) x.k[t] = *reinterpret_cast<const P*>(kp + 4 * t * (D / 2));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pi = __builtin_amdgcn_readlane(page, 4 * i);
    x.v[i] = *reinterpret_cast<const P*>(cache + pi * pb + piece + value_codes<D>(c, (k0 + kCacheChunk * i) & P_mask) + lane * (int)sizeof(P));
  }
  const int sc = (lane >> 3) & 3;
  const int ps = __shfl(page, 4 * sc);
  x.s = *reinterpret_cast<const P*>(cache + ps * pb + piece + scales<D>(c, lane >> 5, (k0 + kCacheChunk * sc) & P_mask) + (lane & 7) * (int)sizeof(P));
}

// The running state of a wave's 16 columns: column lane % 16, and of O^T channels 16 ct + 4h + i.
template <int D>
struct State {
  floatx4v o[D / 16];
  float m, l;
};

// limit: the column's position (its last visible key); unmasked steps are visible to all columns that are rows (the others, q = 0, may
// come to anything: they are dropped).
template <int D, int TERMS, bool MASKED>
__device__ __forceinline__ void step(State<D>& st, const StepData<D>& x, const bf16x8 (&q)[D / 32][TERMS], const char* lds, int k0, int limit,
                                     float scale_log2) {
  constexpr int G = D / 32;
  const int lane = threadIdx.x & 63, h = lane >> 4;
  float s[16];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    // scales of keys 16h + 4t .. +3: G per key
    unsigned sw[2 * G];
    const char* sp = lds + kStep * kVRow<D> + (16 * h + 4 * t) * (D / 16);
#pragma unroll
    for (int i = 0; i < 2 * G; i += 4) {
      const uint4 w = *reinterpret_cast<const uint4*>(sp + 4 * i);
      sw[i] = w.x; sw[i + 1] = w.y; sw[i + 2] = w.z; sw[i + 3] = w.w;
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const bf16x8 a = codes_to_bf16(word(x.k[t], g));
      floatx4v p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = TERMS - 1; n >= 0; --n) p = mfma16(a, q[g][n], p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned w = sw[i * (G / 2) + g / 2];
        const float f = g & 1 ? hi_bf16(w) : lo_bf16(w);
        s[4 * t + i] = g == 0 ? p[i] * f : __builtin_fmaf(p[i], f, s[4 * t + i]);
      }
    }
  }
  if (MASKED) {
    const int last = x.ok >> h & 1 ? limit - k0 - 16 * h : -1;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e > last) s[e] = -INFINITY;
  }
  float mx = s[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  mx *= scale_log2;
  if (__any(mx > st.m)) {
    const float m = fmaxf(st.m, mx), alpha = m == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
    st.m = m;
    st.l *= alpha;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) st.o[ct] *= alpha;
  }
  const float m = st.m == -INFINITY ? 0.f : st.m;            // nothing seen yet: every s is -inf and every probability 0
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale_log2, -m));
    st.l += s[e];
  }
  const char* vs = lds + kStep * kVRow<D> + kScaleBytes<D> + 16 * h * (D / 16);
  const char* vp = lds + lane * kVRow<D>;                    // row 16h + lane % 16 for the transpose reads
#pragma unroll
  for (int gp = 0; gp < G / 2; ++gp) {                       // two scale groups share a word
    unsigned sw[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) sw[e] = *reinterpret_cast<const unsigned*>(vs + e * (D / 16) + 4 * gp);
#pragma unroll
    for (int gi = 0; gi < 2; ++gi) {
      float p[2][8];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float f = gi ? hi_bf16(sw[e]) : lo_bf16(sw[e]);
        p[e >> 3][e & 7] = MASKED && s[e] == 0.f ? 0.f : s[e] * f;   // (a masked key's scale may be anything)
      }
      bf16x8 pt[2][TERMS];
      split_terms<TERMS>(p[0], pt[0]);
      split_terms<TERMS>(p[1], pt[1]);
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        const int ct = 4 * gp + 2 * gi + c2;
        const int2v w = __builtin_amdgcn_ds_read_tr4_b64_v2i32((LDS_PTR(int2v))(vp + 8 * ct));
        const bf16x8 a0 = codes_to_bf16((unsigned)w.x), a1 = codes_to_bf16((unsigned)w.y);
#pragma unroll
        for (int n = TERMS - 1; n >= 0; --n) {
          st.o[ct] = mfma16(a0, pt[0][n], st.o[ct]);
          st.o[ct] = mfma16(a1, pt[1][n], st.o[ct]);
        }
      }
    }
  }
}

// What a sequence contributes to the row of units: its rows, tiles, units per tile.
struct Seq { int row0, rows, len, tiles, units; };

__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int b) {
  Seq s;
  s.row0 = b;
  s.rows = 1;
  if (a.c.row_ptr) {
    s.row0 = min(max(a.c.row_ptr[b], 0), a.c.n_rows);
    s.rows = min(max(a.c.row_ptr[b + 1], s.row0), a.c.n_rows) - s.row0;
  }
  s.len = seq_len(a.c, b);
  s.tiles = (int)(((long long)s.rows * a.group + kCols - 1) / kCols);
  s.units = max(1, (s.len + kUnit - 1) / kUnit);             // rows that see nothing are items too: their outputs are written
  return s;
}
__device__ __forceinline__ long long seq_units(const AttnArgs& a, const Seq& s) { return (long long)s.tiles * s.units * a.c.n_kv_heads; }

__device__ __forceinline__ long long wave_scan(long long x) {   // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = __shfl_up(x, d);
    if ((int)(threadIdx.x & 63) >= d) x += y;
  }
  return x;
}

// Inclusive scan over the block; `total` gets the sum.
__device__ __forceinline__ long long block_scan(long long x, long long* lds, long long& total) {
  x = wave_scan(x);
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[wave] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) x += lds[w];
    total += lds[w];
  }
  return x;
}

// The block that holds unit x of U, when block i of n holds units [U i / n, U (i + 1) / n).
__device__ __forceinline__ int block_of(long long x, long long U, int n) { return (int)(((x + 1) * n - 1) / U); }

template <class T> __device__ __forceinline__ void load_q(const T* p, float sign, float (&x)[8]);
template <> __device__ __forceinline__ void load_q<bf16>(const bf16* p, float sign, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = sign * lo_bf16(word(w, i)); x[2 * i + 1] = sign * hi_bf16(word(w, i)); }
}
template <> __device__ __forceinline__ void load_q<float>(const float* p, float sign, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = sign * p[i];
}

template <int N>
__device__ __forceinline__ void store_out(bf16* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<bf16x4*>(p + i) = bf16x4{(bf16)x[i], (bf16)x[i + 1], (bf16)x[i + 2], (bf16)x[i + 3]};
}
template <int N>
__device__ __forceinline__ void store_out(float* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<floatx4v*>(p + i) = floatx4v{x[i], x[i + 1], x[i + 2], x[i + 3]};
}

template <class T, int D, int TERMS>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(AttnArgs a, const T* __restrict__ q, const char* __restrict__ cache,
                                                                 T* __restrict__ o, float* __restrict__ lse, char* __restrict__ ws) {
  typedef typename Piece<D>::type P;
  __shared__ __align__(16) char lds[kLds<D>];
  __shared__ long long scan[kWaves], found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 4, col = lane & 15;
  const int N = gridDim.x;
  // neighbouring blocks of the row of units on one XCD: tiles of one head read the same keys
  const int id = N % 8 == 0 ? (int)(blockIdx.x % 8) * (N / 8) + blockIdx.x / 8 : blockIdx.x;

  long long U = 0;
  for (int b0 = 0; b0 < a.c.n_seqs; b0 += kThreads) {
    const int b = b0 + tid;
    if (b < a.c.n_seqs) U += seq_units(a, seq_of(a, b));
  }
  long long mine = U;
  mine = block_scan(mine, scan, U);
  const int n = (int)min((long long)N, U);                   // blocks with work: no unit, no block
  if (blockIdx.x == 0 && tid == 0) reinterpret_cast<Header*>(ws)->blocks = n;
  if (id >= n) return;
  const long long u0 = U * id / n, u1 = U * (id + 1) / n;
  long long before = 0;
  for (int b0 = 0;; b0 += kThreads) {                        // ends: u0 < U
    const int b = b0 + tid;
    const long long w = b < a.c.n_seqs ? seq_units(a, seq_of(a, b)) : 0;
    long long total;
    const long long end = before + block_scan(w, scan, total);
    if (u0 < end && u0 >= end - w) { found[0] = b; found[1] = end - w; }
    if (u0 < before + total) break;
    before += total;
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane((int)found[0]);
  long long seq_begin = found[1];
  Split split{0, 0, 0, 0, 0, 0};
  Seq s = seq_of(a, b);

  for (long long u = u0; u < u1;) {
    while (u >= seq_begin + seq_units(a, s)) {               // on to the next sequence with rows
      seq_begin += seq_units(a, s);
      s = seq_of(a, ++b);
    }
    const long long local = u - seq_begin;
    const int item = __builtin_amdgcn_readfirstlane((int)(local / s.units)), first = __builtin_amdgcn_readfirstlane((int)(local % s.units));
    const int last = (int)min((long long)s.units, first + (u1 - u));
    const int hk = item / s.tiles, col0 = (item % s.tiles) * kCols, cols = min(s.rows * a.group - col0, kCols);
    const int base = s.len - s.rows;                         // position of the sequence's row 0
    const int row = (col0 + col) / a.group, head = hk * a.group + (col0 + col) % a.group;
    const bool real = col < cols;
    const int limit = real ? base + row : -1;
    const int visible = base + (col0 + cols - 1) / a.group + 1, all_see = base + col0 / a.group + 1;

    bf16x8 qf[D / 32][TERMS];
    {
      const T* qp = q + ((size_t)(s.row0 + (real ? row : 0)) * a.Hq + (real ? head : 0)) * D + 8 * h;
#pragma unroll
      for (int g = 0; g < D / 32; ++g) {
        float x[8];
        load_q(qp + 32 * g, real ? a.q_sign : 0.f, x);
        if (!real || a.q_sign == 0.f)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
        split_terms<TERMS>(x, qf[g]);
      }
    }
    State<D> st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) st.o[ct] = floatx4v{0.f, 0.f, 0.f, 0.f};

    char* mine_lds = lds + wave * kWaveLds<D>;
    const int end = min(last * kUnit, visible);
    int k0 = first * kUnit + wave * kStep;
    StepData<D> x;
    if (k0 < end) load_step<D>(x, a.c, cache, b, hk, k0, visible);
    for (; k0 < end; k0 += kUnit) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = lane * (int)sizeof(P);                // 16 keys of D/2 bytes
        *reinterpret_cast<P*>(mine_lds + (16 * i + at / (D / 2)) * kVRow<D> + at % (D / 2)) = x.v[i];
      }
      *reinterpret_cast<P*>(mine_lds + kStep * kVRow<D> + (lane >> 5) * kScaleBytes<D> + (lane & 31) * (int)sizeof(P)) = x.s;
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      const StepData<D> now = x;
      if (k0 + kUnit < end) load_step<D>(x, a.c, cache, b, hk, k0 + kUnit, visible);
      if (now.ok == 15 && k0 + kStep <= all_see) step<D, TERMS, false>(st, now, qf, mine_lds, k0, limit, a.scale_log2);
      else step<D, TERMS, true>(st, now, qf, mine_lds, k0, limit, a.scale_log2);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }

    // the four waves' states together
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
    __syncthreads();
    float* ends = reinterpret_cast<float*>(lds);
    float* stat = ends + kWaves * kCols * kOutRow<D>;        // [wave][col] maximum, then sum
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
      *reinterpret_cast<floatx4v*>(ends + (wave * kCols + col) * kOutRow<D> + 16 * ct + 4 * h) = st.o[ct];
    if (h == 0) {
      stat[wave * kCols + col] = st.m;
      stat[kWaves * kCols + wave * kCols + col] = st.l;
    }
    __syncthreads();
    {
      constexpr int E = D / 16;                              // channels of a thread
      const int c = tid >> 4, e0 = (tid & 15) * E;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stat[w * kCols + c]);
      const float ref = m == -INFINITY ? 0.f : m;
      float l = 0.f, out[E];
#pragma unroll
      for (int e = 0; e < E; ++e) out[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(stat[w * kCols + c] - ref);
        l = __builtin_fmaf(stat[kWaves * kCols + w * kCols + c], f, l);
#pragma unroll
        for (int e = 0; e < E; ++e) out[e] = __builtin_fmaf(ends[(w * kCols + c) * kOutRow<D> + e0 + e], f, out[e]);
      }
      if (first == 0 && last == s.units) {
        if (c < cols) {
          const int r = s.row0 + (col0 + c) / a.group, hd = hk * a.group + (col0 + c) % a.group;
          const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
          for (int e = 0; e < E; ++e) out[e] = l == 0.f ? 0.f : out[e] * inv;
          store_out<E>(o + ((size_t)r * a.Hq + hd) * D + e0, out);
          if (lse && e0 == 0) lse[(size_t)hd * a.c.n_rows + r] = (m + __builtin_amdgcn_logf(l)) * kLn2;
        }
      } else {
        float* part = part_of<D>(ws, id, first == 0 ? 1 : 0);
        store_out<E>(part + c * D + e0, out);
        if (e0 == 0) { part[kCols * D + c] = m; part[kCols * D + kCols + c] = l; }
        if (first == 0)
          split = {id, block_of(seq_begin + (long long)item * s.units + s.units - 1, U, n) - id + 1, s.row0, cols, col0, hk * a.group};
      }
    }
    __syncthreads();
    u += last - first;
  }
  if (tid == 0) *reinterpret_cast<Split*>(ws + sizeof(Header) + (size_t)id * 32) = split;
}

// Adds up the parts of the item that block `blockIdx.x` of the first launch began and did not end, column blockIdx.y: 8 runs of parts
// (thread / 32) of four channels each.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache_attn_join_kernel(AttnArgs a, T* __restrict__ o, float* __restrict__ lse, char* __restrict__ ws) {
  constexpr int W = D / 4, R = kThreads / W;                 // threads of a row of D channels; runs
  const int i = blockIdx.x, c = blockIdx.y, tid = threadIdx.x;
  if (i >= reinterpret_cast<const Header*>(ws)->blocks) return;
  const Split s = *reinterpret_cast<const Split*>(ws + sizeof(Header) + (size_t)i * 32);
  if (s.parts == 0 || c >= s.cols) return;
  __shared__ float weight[kMaxGrid], red[kWaves];
  __shared__ float sums[R][D + 4];
  auto part = [&](int p) { return part_of<D>(ws, s.first + p, p == 0 ? 1 : 0); };
  float m = -INFINITY;
  for (int p = tid; p < s.parts; p += kThreads) {
    const float x = part(p)[kCols * D + c];
    weight[p] = x;
    m = fmaxf(m, x);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float ref = m == -INFINITY ? 0.f : m;
  __syncthreads();
  float l = 0.f;
  for (int p = tid; p < s.parts; p += kThreads) {
    const float f = __builtin_amdgcn_exp2f(weight[p] - ref);
    weight[p] = f;
    l = __builtin_fmaf(part(p)[kCols * D + kCols + c], f, l);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
  if ((tid & 63) == 0) red[tid >> 6] = l;
  __syncthreads();
  l = (red[0] + red[1]) + (red[2] + red[3]);
  const int run = tid / W, e = (tid % W) * 4;
  floatx4v x = {0.f, 0.f, 0.f, 0.f};
  for (int p = run; p < s.parts; p += R) x += *reinterpret_cast<const floatx4v*>(part(p) + c * D + e) * weight[p];
  *reinterpret_cast<floatx4v*>(&sums[run][e]) = x;
  __syncthreads();
  if (run != 0) return;
#pragma unroll
  for (int r = 1; r < R; ++r) x += *reinterpret_cast<const floatx4v*>(&sums[r][e]);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float out[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) out[k] = l == 0.f ? 0.f : x[k] * inv;
  const int r = s.row0 + (s.col0 + c) / a.group, hd = s.head0 + (s.col0 + c) % a.group;
  store_out<4>(o + ((size_t)r * a.Hq + hd) * D + e, out);
  if (lse && e == 0) lse[(size_t)hd * a.c.n_rows + r] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Blocks of the first launch: as many as there can be units, up to four per compute unit.
int grid_blocks(const slimattn_cache_params& p, int n_q_heads) {
  const long long cols = (long long)p.n_rows * (n_q_heads / p.n_kv_heads);
  const long long items = (cols / kCols + p.n_seqs) * p.n_kv_heads;
  const long long units = ((long long)p.max_pages * p.page_size + kUnit - 1) / kUnit;
  const long long most = items > kMaxGrid ? kMaxGrid : items * units;
  return (int)(most < kMaxGrid ? most : kMaxGrid);
}

}  // namespace

CacheView cache_view(const slimattn_cache_params& p, const int32_t* row_ptr, const int32_t* lens, const int32_t* table);

size_t cache_attn_bytes(const slimattn_cache_params& p, int n_q_heads) {
  const size_t part = (size_t)(kCols * p.head_dim + 2 * kCols) * sizeof(float);
  return sizeof(Header) + (size_t)kMaxGrid * 32 + (size_t)grid_blocks(p, n_q_heads) * 2 * part;
}

int launch_cache_attn(const slimattn_cache_params& p, int n_q_heads, float scale, const void* q, const int32_t* row_ptr, const int32_t* lens,
                      const int32_t* table, const void* cache, void* o, float* lse, void* ws, void* stream) {
  AttnArgs a{cache_view(p, row_ptr, lens, table), n_q_heads / p.n_kv_heads, n_q_heads, 0.f, 1.f};
  const float f = scale * 1.4426950408889634f, size = f < 0.f ? -f : f;
  a.q_sign = f < 0.f ? -1.f : f > 0.f ? 1.f : 0.f;
  a.scale_log2 = size > 0x1p-126f ? size : 0x1p-126f;        // masked scores are -inf times it
  const int blocks = grid_blocks(p, n_q_heads);
  auto run = [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, TERMS = sizeof(T) == 4 ? 3 : 1;
    hipLaunchKernelGGL((cache_attn_kernel<T, D, TERMS>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)q, (const char*)cache,
                       (T*)o, lse, (char*)ws);
    const int e = (int)hipGetLastError();
    if (e != 0 || blocks < 2) return e;                      // one block holds every item whole
    hipLaunchKernelGGL((cache_attn_join_kernel<T, D>), dim3((unsigned)blocks, kCols), dim3(kThreads), 0, (hipStream_t)stream, a, (T*)o, lse, (char*)ws);
    return (int)hipGetLastError();
  };
  if (p.dtype == SLIMATTN_F32) return p.head_dim == 128 ? run(float{}, IC<128>{}) : run(float{}, IC<64>{});
  return p.head_dim == 128 ? run(bf16{}, IC<128>{}) : run(bf16{}, IC<64>{});
}

}  // namespace slimattn
