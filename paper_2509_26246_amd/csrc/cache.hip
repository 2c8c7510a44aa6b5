// Quantising keys and values into the pages of a 4-bit cache, and reading rows back (layout: cache.h).
//
// Mathematics.  Of 32 channels, a = max |x|; scale s = a / 6 rounded to six significant bits (ties to even); code = the nearest of the 4-bit
// floats to x / s, ties to the even code.  Both roundings are those of the real quotients: a / 6 is a correctly rounded 32-bit quotient, and
// so is x / s here (product with 1 / s, one exact remainder, one correction).  A correctly rounded quotient is at a border between two codes only if the
// real one is: borders have three bits and s six, so border * s is itself a 24-bit number; an x beside it is off by a whole step, and its quotient by more than
// half a step of the border's.
//
// Bound by memory and latency: 2 bytes in, 0.56 out for a bf16 value (and back).  A lane takes eight channels (16 bytes of bf16, one word of codes), four lanes
// share a scale by two lane exchanges; a wave stays with one row, whose page it looks up once.  Measured, bf16, 8 heads of 128: 10764 rows (57 MB either
// way) 13.3 us written, 11.8 read (4.3 and 4.8 TB/s); 21188 rows read 20.0 us (5.6 TB/s); 64 rows 3.0 us, a launch's latency.
#include <hip/hip_runtime.h>

#include "cache.h"

namespace slimattn {
namespace {

constexpr int kThreads = 256;

// parts: waves that share a row's 2 * Hkv head rows (keys and values of each head).
struct CopyArgs { CacheView c; int parts; long long k_stride, v_stride; };

template <class T> __device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<bf16>(const bf16* p, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = lo_bf16(u[i]); x[2 * i + 1] = hi_bf16(u[i]); }
}
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const floatx4 a = *reinterpret_cast<const floatx4*>(p), b = *reinterpret_cast<const floatx4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
// Rows read back are streamed past the caches: 21188 rows of 8 heads of 128 30.0 -> 21.0 us among other work; slimattn_fwd behind it within 0.5%.
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (bf16)x[i];
  __builtin_nontemporal_store(v, reinterpret_cast<bf16x8*>(p));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  __builtin_nontemporal_store(floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<floatx4*>(p));
  __builtin_nontemporal_store(floatx4{x[4], x[5], x[6], x[7]}, reinterpret_cast<floatx4*>(p + 4));
}

// The scale of 32 channels from the largest |x| (its bits: infinities and NaN are the largest).  Below 2^-100 a group is zero (its
// codes' arithmetic would leave the normal numbers), above the scale is kept where six times it is finite; an infinity or a NaN makes the
// scale, and with it all 32 values, NaN.
__device__ __forceinline__ float group_scale(unsigned a) {
  const float six = __builtin_bit_cast(float, a) / 6.f;
  unsigned u = __builtin_bit_cast(unsigned, six);
  u = (u + 0x1ffffu + ((u >> 18) & 1u)) & 0xfffc0000u;
  u = min(u, 0x7e280000u);                                   // 1.3125 * 2^125
  if (a < 0x0d800000u) u = 0;                                // 2^-100
  if (a >= 0x7f800000u) u = 0x7fc00000u;
  return __builtin_bit_cast(float, u);
}

__device__ __forceinline__ unsigned encode8(const float (&x)[8], float s) {
  const float r = s != 0.f ? 1.f / s : 0.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = x[i] * r;
    y[i] = __builtin_fmaf(__builtin_fmaf(-q, s, x[i]), r, q);
  }
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
  return w;
}

// Where this wave works: its row, the page piece of the row's token, and the head rows [first, last) of 2 * Hkv it takes.
struct Place { bool any; int row, page, token, first, last; };

__device__ __forceinline__ Place wave_place(const CopyArgs& a) {
  const long long wave = (long long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Place p;
  p.any = wave < (long long)a.c.n_rows * a.parts;
  if (!p.any) return p;
  p.row = (int)(wave / a.parts);
  const int part = (int)(wave % a.parts), n = 2 * a.c.n_kv_heads, each = (n + a.parts - 1) / a.parts;
  p.first = part * each;
  p.last = min(p.first + each, n);
  const int b = wave_find_seq(a.c, p.row), pos = row_position(a.c, p.row, b);
  p.any = pos != INT32_MIN;
  p.page = pos >= 0 ? page_at(a.c, b, pos) : -1;
  p.token = pos & ((1 << a.c.page_shift) - 1);
  return p;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CopyArgs a, const T* __restrict__ k, const T* __restrict__ v, char* __restrict__ cache) {
  constexpr int L = D / 8, R = 64 / L, G = D / kCacheGroup;
  const Place p = wave_place(a);
  if (!p.any || p.page < 0) return;
  const int lane = threadIdx.x & 63, j = lane % L;
  char* page = cache + p.page * page_bytes<D>(a.c);
  for (int i = p.first + lane / L; i < p.last; i += R) {     // keys and values of a head in turn; groups of four lanes stay together
    const int h = i >> 1, value = i & 1;
    float x[8];
    load8((value ? v + p.row * a.v_stride : k + p.row * a.k_stride) + (size_t)h * D + 8 * j, x);
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __builtin_bit_cast(unsigned, x[e]) & 0x7fffffffu);
    m = max(m, (unsigned)__shfl_xor((int)m, 1));
    m = max(m, (unsigned)__shfl_xor((int)m, 2));
    const float s = group_scale(m);
    const unsigned w = encode8(x, s);
    char* piece = page + h * head_bytes<D>(a.c);
    const int at = value ? value_codes<D>(a.c, p.token) + 4 * j : key_codes<D>(p.token) + 4 * ((j & 3) * G + (j >> 2));
    *reinterpret_cast<unsigned*>(piece + at) = w;
    if ((j & 3) == 0)
      *reinterpret_cast<unsigned short*>(piece + scales<D>(a.c, value, p.token) + 2 * (j >> 2)) = (unsigned short)(__builtin_bit_cast(unsigned, s) >> 16);
  }
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CopyArgs a, const char* __restrict__ cache, T* __restrict__ k, T* __restrict__ v) {
  constexpr int L = D / 8, R = 64 / L, G = D / kCacheGroup;
  const Place p = wave_place(a);
  if (!p.any) return;
  const int lane = threadIdx.x & 63, j = lane % L;
  const char* page = cache + max(p.page, 0) * page_bytes<D>(a.c);
  for (int i = p.first + lane / L; i < p.last; i += R) {
    const int h = i >> 1, value = i & 1;
    float x[8];
    if (p.page >= 0) {
      const char* piece = page + h * head_bytes<D>(a.c);
      const int at = value ? value_codes<D>(a.c, p.token) + 4 * j : key_codes<D>(p.token) + 4 * ((j & 3) * G + (j >> 2));
      const bf16x8 codes = codes_to_bf16(*reinterpret_cast<const unsigned*>(piece + at));
      const unsigned short s16 = *reinterpret_cast<const unsigned short*>(piece + scales<D>(a.c, value, p.token) + 2 * (j >> 2));
      const float s = __builtin_bit_cast(float, (unsigned)s16 << 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s * (float)codes[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
    }
    store8((value ? v : k) + ((size_t)p.row * a.c.n_kv_heads + h) * D + 8 * j, x);
  }
}

// A row's head rows stay with one wave unless there are too few rows to give every SIMD two waves.
int row_parts(int n_rows, int n_kv_heads, int d) {
  const long long most = (2 * n_kv_heads + 512 / d - 1) / (512 / d), want = (2048 + n_rows - 1) / n_rows;   // 512 / d head rows fill a wave
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

template <class F>
int by_type(int dtype, int d, F&& f) {
  if (dtype == SLIMATTN_F32) return d == 128 ? f(float{}, IC<128>{}) : f(float{}, IC<64>{});
  return d == 128 ? f(bf16{}, IC<128>{}) : f(bf16{}, IC<64>{});
}

}  // namespace

CacheView cache_view(const slimattn_cache_params& p, const int32_t* row_ptr, const int32_t* lens, const int32_t* table) {
  int shift = 0;
  while ((1 << shift) < p.page_size) ++shift;
  return {p.n_pages, shift, p.n_kv_heads, p.n_seqs, p.max_pages, p.n_rows, p.max_pages * p.page_size, row_ptr, lens, table};
}

int launch_cache_write(const slimattn_cache_params& p, const void* k, const void* v, int64_t k_stride, int64_t v_stride, const int32_t* row_ptr,
                       const int32_t* lens, const int32_t* table, void* cache, void* stream) {
  const int parts = row_parts(p.n_rows, p.n_kv_heads, p.head_dim);
  const CopyArgs a{cache_view(p, row_ptr, lens, table), parts, k_stride, v_stride};
  const long long blocks = ((long long)p.n_rows * parts + 3) / 4;
  return by_type(p.dtype, p.head_dim, [&](auto t, auto d) {
    using T = decltype(t);
    hipLaunchKernelGGL((cache_write_kernel<T, decltype(d)::value>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)k,
                       (const T*)v, (char*)cache);
    return (int)hipGetLastError();
  });
}

int launch_cache_read(const slimattn_cache_params& p, const void* cache, const int32_t* row_ptr, const int32_t* lens, const int32_t* table, void* k,
                      void* v, void* stream) {
  const int parts = row_parts(p.n_rows, p.n_kv_heads, p.head_dim);
  const CopyArgs a{cache_view(p, row_ptr, lens, table), parts, 0, 0};
  const long long blocks = ((long long)p.n_rows * parts + 3) / 4;
  return by_type(p.dtype, p.head_dim, [&](auto t, auto d) {
    using T = decltype(t);
    hipLaunchKernelGGL((cache_read_kernel<T, decltype(d)::value>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const char*)cache,
                       (T*)k, (T*)v);
    return (int)hipGetLastError();
  });
}

}  // namespace slimattn
