// Queries and keys before attention: norm per head and rotation by the token's positions in one pass, and the gradients of both.
//
// Mathematics.  A head's row x of d channels: r = 1 / sqrt(mean x^2 + eps), n = x r w; pair (a, b) of n turns by t = position * frequency.
// Backwards, with g the gradient turned by -t: dw = sum over tokens and heads of g x r; h = g w; dx = r (h - x r^2 mean(h x)).  r is
// computed again from x, which has to be read for dw in any case, so the forward pass stores nothing for the backward.  The weights' sums are fp32 throughout, a
// few rows per lane and then a tree: 2e-7 of the gradient's norm from 1.3 million terms (added in 64 bits 0.8e-7, the terms' own rounding).
//
// Bound by memory: the forward reads and writes each element once, the backward reads x and dy and writes dx.  So that a pass needs no
// exchange but the sum of squares, a lane holds two runs of four channels that contain both halves of its four pairs, whichever way
// pairs are formed: channels 4j .. 4j+3 and rotary/2 + 4j .. (8 j .. 8j+7 where neighbours pair up, or behind the rotated channels).
// Measured: 32768 tokens of 32 + 8 heads of 128, bf16: forward 129 us (0.67 GB, 5.2 TB/s; a large copy reaches 4.9), backward 213 us (1.0 GB, 4.7 TB/s) and 3 to 5
// for the weights' sums; 4099 tokens of 8 + 2 heads, fp32: 10 and 13 us; 16 tokens of 32 + 8 heads, forward: 4.2 us, launch and one walk's latency.
// A head takes d/8 lanes, a wave 64 / (d/8) heads; the lanes of one head ("group") keep a token and walk its heads, so the four
// sines and cosines of a lane are computed once per token and not once per head.  Few tokens are divided by heads as well.
//
// Angles: position * frequency (31 x 24 bits) and its turns are formed exactly, as two 64-bit numbers, and reduced to a quarter turn around zero before they
// are rounded to 32 bits, so that far positions lose nothing: in 32 bits a position of 10^6 would be off by 0.03 rad, in one 64-bit number one of 2^31
// by 4e-7, several times what rounding the reduced angle costs.  Sine and cosine of at most pi/4 are their Taylor sums (the first term left
// out is below 2e-9), which costs less than the general functions' own reduction.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "mfma_utils.h"

namespace slimattn {
namespace {

constexpr int kThreads = 256;
constexpr int kBwdBlocks = 1024;   // backward blocks: each leaves one partial sum of the weights' gradients

template <int D> constexpr int kLanes = D / 8;                 // lanes of a head
template <int D> constexpr int kGroups = kThreads / kLanes<D>; // groups of a block

// What a lane reads and writes of a head row: four channels from c0, four from c1.  Pairs p(0..3): see turn().
struct Chan { int c0, c1; bool rotated; };

template <bool ADJ>
__device__ __forceinline__ Chan lane_channels(int j, int rotary) {
  const int in_turn = rotary >> 3;
  if (ADJ || j >= in_turn) return {8 * j, 8 * j + 4, j < in_turn};
  return {4 * j, (rotary >> 1) + 4 * j, true};
}

// The number of the i-th pair of lane j (all of a lane's pairs are neighbours).
__device__ __forceinline__ int first_pair(int j) { return 4 * j; }

struct Turn { float c[4], s[4]; };

// Sine and cosine of pos * freq.  u + lo: turns (the product with its remainder, times 1 / 2 pi in two words: off by less than 2^-100 of them); their fraction
// is reduced to an eighth around the nearest quarter turn.
__device__ __forceinline__ void turn_of(int pos, float freq, float& c, float& s) {
#pragma clang fp contract(off)   // (u itself is what lo completes)
  constexpr double kTurn = 0.15915494309189535, kTurnLow = -9.839338337591243e-18;
  const double p = (double)pos * (double)freq, u = p * kTurn;
  const double lo = __builtin_fma(__builtin_fma((double)pos, (double)freq, -p), kTurn, __builtin_fma(p, kTurnLow, __builtin_fma(p, kTurn, -u)));
  double f = (u - __builtin_rint(u)) + lo;
  f -= __builtin_rint(f);
  const double k = __builtin_rint(4.0 * f);
  const float a = (float)((f - 0.25 * k) * 6.283185307179586477);
  const int quarter = (int)k & 3;
  const float a2 = a * a;
  const float sn = __builtin_fmaf(a * a2, __builtin_fmaf(a2, __builtin_fmaf(a2, __builtin_fmaf(a2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), a);
  const float cs = __builtin_fmaf(a2, __builtin_fmaf(a2, __builtin_fmaf(a2, __builtin_fmaf(a2, __builtin_fmaf(a2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float x = quarter & 1 ? sn : cs, y = quarter & 1 ? cs : sn;
  c = (quarter == 1 || quarter == 2) ? -x : x;
  s = quarter & 2 ? -y : y;
}

// axes: two bits per pair, pairs 0..31 and 32..63.
struct RopeArgs {
  int T, Hq, Hk, rotary;
  int heads_per_item, items_per_token;
  unsigned long long axes[2];
  float eps;
  long long q_stride, k_stride, dq_stride, dk_stride;
};

__device__ __forceinline__ void load_turns(Turn& t, const RopeArgs& a, const Chan& ch, int j, int token, const int32_t* __restrict__ positions,
                                           const float* __restrict__ inv_freq) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { t.c[i] = 1.f; t.s[i] = 0.f; }
  if (!ch.rotated) return;
  const int p0 = first_pair(j);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = p0 + i, axis = (int)(a.axes[p >> 5] >> (2 * (p & 31))) & 3;
    turn_of(positions[(size_t)axis * a.T + token], inv_freq[p], t.c[i], t.s[i]);
  }
}

// x[0..3] = channels c0.., x[4..7] = channels c1..; by `sign` forwards (+1) or back (-1).
template <bool ADJ>
__device__ __forceinline__ void turn(float (&x)[8], const Turn& t, float sign) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int ia = ADJ ? 2 * i : i, ib = ADJ ? 2 * i + 1 : i + 4;
    const float a = x[ia], b = x[ib], s = sign * t.s[i];
    x[ia] = a * t.c[i] - b * s;
    x[ib] = b * t.c[i] + a * s;
  }
}

typedef unsigned int uint2v __attribute__((ext_vector_type(2)));

// One lane's eight elements of a row, as they are in memory.
template <class T> struct Raw;
template <> struct Raw<bf16> { uint2v a, b; };
template <> struct Raw<float> { floatx4 a, b; };

template <class T>
__device__ __forceinline__ Raw<T> load_row(const T* row, const Chan& ch) {
  Raw<T> r;
  r.a = *reinterpret_cast<const decltype(r.a)*>(row + ch.c0);
  r.b = *reinterpret_cast<const decltype(r.b)*>(row + ch.c1);
  return r;
}
__device__ __forceinline__ void widen(const Raw<bf16>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[2 * i] = __builtin_bit_cast(float, r.a[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, r.a[i] & 0xffff0000u);
    x[4 + 2 * i] = __builtin_bit_cast(float, r.b[i] << 16);
    x[4 + 2 * i + 1] = __builtin_bit_cast(float, r.b[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const Raw<float>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = r.a[i]; x[4 + i] = r.b[i]; }
}
// Outputs are streamed past the caches: 32768 tokens both ways 358 -> 353 us, 4099 tokens in fp32 28.6 -> 26.4; slimattn_fwd behind it takes what it
// took (512 to 32768 tokens, within 0.5%).  Streaming the loads as well costs a backward soon after its forward the second reading (26.4 -> 37.4).
__device__ __forceinline__ void store_row(bf16* row, const Chan& ch, const float (&x)[8]) {
  const bf16x4 a = {(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]}, b = {(bf16)x[4], (bf16)x[5], (bf16)x[6], (bf16)x[7]};
  __builtin_nontemporal_store(a, reinterpret_cast<bf16x4*>(row + ch.c0));
  __builtin_nontemporal_store(b, reinterpret_cast<bf16x4*>(row + ch.c1));
}
__device__ __forceinline__ void store_row(float* row, const Chan& ch, const float (&x)[8]) {
  __builtin_nontemporal_store(floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<floatx4*>(row + ch.c0));
  __builtin_nontemporal_store(floatx4{x[4], x[5], x[6], x[7]}, reinterpret_cast<floatx4*>(row + ch.c1));
}

// 1 / sqrt(a), a >= 2^-100: the instruction's last bit corrected by one Newton step.
__device__ __forceinline__ float inv_sqrt(float a) {
  const float r = __builtin_amdgcn_rsqf(a);
  return __builtin_fmaf(0.5f * r, __builtin_fmaf(-a * r, r, 1.f), r);
}

template <int L>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int m = 1; m < L; m <<= 1) x += __shfl_xor(x, m);
  return x;
}

__device__ __forceinline__ void load_weight(float (&w)[8], const float* __restrict__ weight, const Chan& ch) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { w[i] = weight ? weight[ch.c0 + i] : 1.f; w[4 + i] = weight ? weight[ch.c1 + i] : 1.f; }
}

// Heads [h0, h1) of one token, four rows in flight.
template <class T, int D, bool NORM, bool ADJ>
__device__ __forceinline__ void fwd_heads(const T* src, T* dst, int h0, int h1, const Chan& ch, const Turn& t, const float (&w)[8], float eps) {
  constexpr int U = 4;
  for (int h = h0; h < h1; h += U) {
    Raw<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = load_row(src + (size_t)min(h + u, h1 - 1) * D, ch);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      widen(raw[u], x);
      if (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
        const float r = inv_sqrt(__builtin_fmaf(group_sum<kLanes<D>>(ss), 1.f / D, eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
      }
      turn<ADJ>(x, t, 1.f);
      if (h + u < h1) store_row(dst + (size_t)(h + u) * D, ch, x);
    }
  }
}

template <class T, int D, bool NORM, bool ADJ>
__global__ __launch_bounds__(kThreads) void rope_fwd_kernel(RopeArgs a, const T* q, const T* k, const float* __restrict__ qw,
                                                            const float* __restrict__ kw, const int32_t* __restrict__ positions,
                                                            const float* __restrict__ inv_freq, T* q_out, T* k_out) {
  const int j = threadIdx.x % kLanes<D>, H = a.Hq + a.Hk;
  const long long item = (long long)blockIdx.x * kGroups<D> + threadIdx.x / kLanes<D>;
  const long long token_l = item / a.items_per_token;
  if (token_l >= a.T) return;                              // whole groups leave: the sums below stay within a group
  const int token = (int)token_l, h0 = (int)(item % a.items_per_token) * a.heads_per_item, h1 = min(h0 + a.heads_per_item, H);
  const Chan ch = lane_channels<ADJ>(j, a.rotary);
  Turn t;
  load_turns(t, a, ch, j, token, positions, inv_freq);
  float w[8];
  if (h0 < a.Hq) {
    if (NORM) load_weight(w, qw, ch);
    fwd_heads<T, D, NORM, ADJ>(q + (size_t)token * a.q_stride, q_out + (size_t)token * a.Hq * D, h0, min(h1, a.Hq), ch, t, w, a.eps);
  }
  if (h1 > a.Hq) {
    if (NORM) load_weight(w, kw, ch);
    fwd_heads<T, D, NORM, ADJ>(k + (size_t)token * a.k_stride, k_out + (size_t)token * a.Hk * D, max(h0 - a.Hq, 0), h1 - a.Hq, ch, t, w, a.eps);
  }
}

template <class T, int D, bool NORM, bool ADJ>
__device__ __forceinline__ void bwd_heads(const T* x_row, const T* g_row, T* dst, int h0, int h1, const Chan& ch, const Turn& t,
                                          const float (&w)[8], float (&dw)[8], float eps) {
  constexpr int U = NORM ? 2 : 4;
  for (int h = h0; h < h1; h += U) {
    Raw<T> xr[U], gr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t off = (size_t)min(h + u, h1 - 1) * D;
      gr[u] = load_row(g_row + off, ch);
      if (NORM) xr[u] = load_row(x_row + off, ch);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float g[8];
      widen(gr[u], g);
      turn<ADJ>(g, t, -1.f);
      if (NORM) {
        float x[8], ss = 0.f, hx = 0.f;
        widen(xr[u], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          ss = __builtin_fmaf(x[i], x[i], ss);
          hx = __builtin_fmaf(g[i] * w[i], x[i], hx);
        }
        ss = group_sum<kLanes<D>>(ss);
        hx = group_sum<kLanes<D>>(hx);
        const float r = inv_sqrt(__builtin_fmaf(ss, 1.f / D, eps)), m = hx * (1.f / D) * r * r;
        const bool real = h + u < h1;                      // the row read again in place of one past the end adds nothing
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dw[i] = real ? __builtin_fmaf(g[i] * r, x[i], dw[i]) : dw[i];
          g[i] = r * (g[i] * w[i] - x[i] * m);
        }
      }
      if (h + u < h1) store_row(dst + (size_t)(h + u) * D, ch, g);
    }
  }
}

// A block's partial sum of the weights' gradients: partial[block][query, key][D].
template <class T, int D, bool NORM, bool ADJ>
__global__ __launch_bounds__(kThreads) void rope_bwd_kernel(RopeArgs a, const T* q, const T* k, const float* __restrict__ qw,
                                                            const float* __restrict__ kw, const int32_t* __restrict__ positions,
                                                            const float* __restrict__ inv_freq, const T* gq, const T* gk, T* dq, T* dk,
                                                            float* __restrict__ partial) {
  const int j = threadIdx.x % kLanes<D>, group = threadIdx.x / kLanes<D>, H = a.Hq + a.Hk;
  const Chan ch = lane_channels<ADJ>(j, a.rotary);
  float wq[8], wk[8], dwq[8], dwk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dwq[i] = dwk[i] = 0.f;
  if (NORM && a.Hq) load_weight(wq, qw, ch);
  if (NORM && a.Hk) load_weight(wk, kw, ch);
  const long long items = (long long)a.T * a.items_per_token, step = (long long)gridDim.x * kGroups<D>;
  for (long long item = (long long)blockIdx.x * kGroups<D> + group; item < items; item += step) {
    const int token = (int)(item / a.items_per_token), h0 = (int)(item % a.items_per_token) * a.heads_per_item, h1 = min(h0 + a.heads_per_item, H);
    Turn t;
    load_turns(t, a, ch, j, token, positions, inv_freq);
    if (h0 < a.Hq)
      bwd_heads<T, D, NORM, ADJ>(q + (size_t)token * a.q_stride, gq + (size_t)token * a.Hq * D, dq + (size_t)token * a.dq_stride, h0, min(h1, a.Hq),
                                 ch, t, wq, dwq, a.eps);
    if (h1 > a.Hq)
      bwd_heads<T, D, NORM, ADJ>(k + (size_t)token * a.k_stride, gk + (size_t)token * a.Hk * D, dk + (size_t)token * a.dk_stride, max(h0 - a.Hq, 0),
                                 h1 - a.Hq, ch, t, wk, dwk, a.eps);
  }
  if (!NORM || !partial) return;
  // groups of a wave by lane exchange, the four waves through LDS, in that order
  __shared__ float sums[kThreads / 64][2 * D];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int m = kLanes<D>; m < 64; m <<= 1) {
      dwq[i] += __shfl_xor(dwq[i], m);
      dwk[i] += __shfl_xor(dwk[i], m);
    }
    const int c = i < 4 ? ch.c0 + i : ch.c1 + i - 4;
    if ((threadIdx.x & 63) < kLanes<D>) {
      sums[threadIdx.x >> 6][c] = dwq[i];
      sums[threadIdx.x >> 6][D + c] = dwk[i];
    }
  }
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += sums[w][threadIdx.x];
    partial[(size_t)blockIdx.x * 2 * D + threadIdx.x] = s;
  }
}

// dq_weight[c], dk_weight[c] = sum over blocks of partial[block][..][c]: 16 columns per block, 64 strided sums of each, added in a fixed order.
// The partial sums lie behind another launch's stores, a microsecond away: all of a thread's loads, 16 at most, are on their way at once: 3 to 5 us (16
// sums of 64 loads one after the other: 21).
constexpr int kWeightRuns = 64;
__global__ __launch_bounds__(16 * kWeightRuns) void rope_weight_kernel(const float* __restrict__ partial, int n_blocks, int D, float* dqw, float* dkw) {
  __shared__ float sums[kWeightRuns][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float x[kBwdBlocks / kWeightRuns], s = 0.f;
#pragma unroll
  for (int i = 0; i < kBwdBlocks / kWeightRuns; ++i) {
    const int b = r + i * kWeightRuns;
    x[i] = b < n_blocks ? partial[(size_t)b * 2 * D + col] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kBwdBlocks / kWeightRuns; ++i) s += x[i];
  sums[r][c] = s;
  __syncthreads();
  if (r != 0) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kWeightRuns; ++i) s += sums[i][c];
  float* out = col < D ? dqw : dkw;
  if (out) out[col < D ? col : col - D] = s;
}

// Items: one token's heads [h0, h0 + heads_per_item).  The heads of a token stay together (its angles are computed once) unless there
// are too few tokens to give every SIMD two waves; then they are divided as far as single heads.
RopeArgs make_args(const slimattn_rope_params& p) {
  RopeArgs a{};
  const int H = p.n_q_heads + p.n_kv_heads, d = p.head_dim;
  a.T = p.total_tokens; a.Hq = p.n_q_heads; a.Hk = p.n_kv_heads; a.rotary = p.rotary_dim; a.eps = p.eps;
  const long long want = 2048ll * 64 / (d / 8);            // groups for 256 x 4 SIMDs, two waves each
  long long parts = a.T > 0 ? (want + a.T - 1) / a.T : 1;
  parts = parts < 1 ? 1 : parts > H ? H : parts;
  a.heads_per_item = (int)((H + parts - 1) / parts);
  a.items_per_token = (H + a.heads_per_item - 1) / a.heads_per_item;
  a.q_stride = p.q_stride ? p.q_stride : (long long)p.n_q_heads * d;
  a.k_stride = p.k_stride ? p.k_stride : (long long)p.n_kv_heads * d;
  a.dq_stride = p.dq_stride ? p.dq_stride : (long long)p.n_q_heads * d;
  a.dk_stride = p.dk_stride ? p.dk_stride : (long long)p.n_kv_heads * d;
  int left[4] = {0, 0, 0, 0}, axis = 0;
  for (int i = 0; p.rotary_dim > 0 && i < p.n_axes; ++i) left[i] = p.sections[i];   // (n_axes is checked where there is a rotation)
  for (int i = 0; i < p.rotary_dim / 2; ++i) {             // sections add up to the number of pairs
    while (left[axis] == 0) axis = (axis + 1) & 3;
    --left[axis];
    a.axes[i >> 5] |= (unsigned long long)axis << (2 * (i & 31));
    if (p.flags & SLIMATTN_ROPE_DEALT) axis = (axis + 1) & 3;
  }
  return a;
}

template <int D>
int bwd_blocks(const RopeArgs& a) {
  const long long n = ((long long)a.T * a.items_per_token + kGroups<D> - 1) / kGroups<D>;
  return (int)(n < kBwdBlocks ? n : kBwdBlocks);
}

template <class F>
int by_dim(int d, F&& f) {
  switch (d) {
    case 16: return f(IC<16>{});
    case 32: return f(IC<32>{});
    case 64: return f(IC<64>{});
    default: return f(IC<128>{});
  }
}

template <class T, bool NORM, bool ADJ>
int launch_fwd(const slimattn_rope_params& p, const void* q, const void* k, const float* qw, const float* kw, const int32_t* pos,
               const float* freq, void* qo, void* ko, void* stream) {
  const RopeArgs a = make_args(p);
  return by_dim(p.head_dim, [&](auto d) {
    constexpr int D = decltype(d)::value;
    const long long blocks = ((long long)a.T * a.items_per_token + kGroups<D> - 1) / kGroups<D>;
    hipLaunchKernelGGL((rope_fwd_kernel<T, D, NORM, ADJ>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)q, (const T*)k,
                       qw, kw, pos, freq, (T*)qo, (T*)ko);
    return (int)hipGetLastError();
  });
}

template <class T, bool NORM, bool ADJ>
int launch_bwd(const slimattn_rope_params& p, const void* q, const void* k, const float* qw, const float* kw, const int32_t* pos,
               const float* freq, const void* gq, const void* gk, void* dq, void* dk, float* dqw, float* dkw, void* ws, void* stream) {
  const RopeArgs a = make_args(p);
  return by_dim(p.head_dim, [&](auto d) {
    constexpr int D = decltype(d)::value;
    const int blocks = bwd_blocks<D>(a);
    const bool weights = NORM && (dqw || dkw);
    if (blocks > 0) {
      hipLaunchKernelGGL((rope_bwd_kernel<T, D, NORM, ADJ>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)q, (const T*)k,
                         qw, kw, pos, freq, (const T*)gq, (const T*)gk, (T*)dq, (T*)dk, weights ? (float*)ws : nullptr);
      const int e = (int)hipGetLastError();
      if (e != 0) return e;
    }
    if (!weights) return 0;
    hipLaunchKernelGGL(rope_weight_kernel, dim3(2 * D / 16), dim3(16 * kWeightRuns), 0, (hipStream_t)stream, (const float*)ws, blocks, D, dqw, dkw);
    return (int)hipGetLastError();
  });
}

template <class F>
int by_kind(const slimattn_rope_params& p, F&& f) {
  const bool norm = p.flags & SLIMATTN_ROPE_NORM, adj = p.flags & SLIMATTN_ROPE_ADJACENT;
  auto with = [&](auto t) {
    using T = decltype(t);
    return norm ? (adj ? f(T{}, IC<1>{}, IC<1>{}) : f(T{}, IC<1>{}, IC<0>{})) : (adj ? f(T{}, IC<0>{}, IC<1>{}) : f(T{}, IC<0>{}, IC<0>{}));
  };
  return p.dtype == SLIMATTN_F32 ? with(float{}) : with(bf16{});
}

}  // namespace

// The same for any number of tokens, so that one workspace serves calls of all sizes.
size_t rope_partial_bytes(const slimattn_rope_params& p) { return (size_t)kBwdBlocks * 2 * p.head_dim * sizeof(float); }

int launch_rope_fwd(const slimattn_rope_params& p, const void* q, const void* k, const float* qw, const float* kw, const int32_t* pos,
                    const float* freq, void* qo, void* ko, void* stream) {
  return by_kind(p, [&](auto t, auto norm, auto adj) {
    return launch_fwd<decltype(t), decltype(norm)::value != 0, decltype(adj)::value != 0>(p, q, k, qw, kw, pos, freq, qo, ko, stream);
  });
}

int launch_rope_bwd(const slimattn_rope_params& p, const void* q, const void* k, const float* qw, const float* kw, const int32_t* pos,
                    const float* freq, const void* gq, const void* gk, void* dq, void* dk, float* dqw, float* dkw, void* ws, void* stream) {
  return by_kind(p, [&](auto t, auto norm, auto adj) {
    return launch_bwd<decltype(t), decltype(norm)::value != 0, decltype(adj)::value != 0>(p, q, k, qw, kw, pos, freq, gq, gk, dq, dk, dqw, dkw, ws, stream);
  });
}

}  // namespace slimattn
