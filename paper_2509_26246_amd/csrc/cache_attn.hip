// Attention of each sequence's last rows over its 4-bit cache (layout: cache.h), few rows per sequence: single tokens, drafted tokens.
//
// Mathematics.  S = K q over the codes: the 32 channels of a scale group are one 16x16x32 product, whose 16 keys x 16 query columns are then
// multiplied by the keys' scales in fp32 and added up over the groups: no value of K is ever formed, and q enters as it is.  Likewise
// O^T = V^T P^T takes V's codes as they are, and the probabilities of a scale group times that group's scales.
// Softmax statistics and sums are fp32, in log2 units; the maximum moves with every step.
//
// Fewer bits.  bf16 calls round probability times scale to bf16, the only rounding beside the output's: at most 2^-8 of each term, with either sign, so that an
// output is off by 2.3e-3 of itself where rounding it alone costs 1.65e-3.  A second bf16 term of P (16 bits) gives 1.65e-3 and takes a product more and the
// packing: 64 sequences of up to 4096 keys, 32 heads over 8, 53.6 -> 64.6 us, four of 131072 30.9 -> 36.4.  Not taken: slimattn_fwd rounds P
// alike.  fp32 calls hand q and P over as three bf16 terms, 24 bits: with exact codes the products are then as good as fp32 ones.
//
// Bound by memory (144 bytes per key and KV head at head dim 128 against 4 * 128 flops per query head), so what counts is that every compute unit reads
// all the time, whatever the lengths are.  The columns of a sequence's KV head (rows x heads of the group) are cut into tiles of 16, an item is
// one tile's walk over the keys it sees, its length counted in units of 256 keys; the units of all items in a row are divided evenly among
// the blocks of one launch, which find their place in that row by a scan over the lengths (they are data: a recorded call follows
// them).  A block's first and last item may be parts; parts leave O, maximum and sum in the workspace, and a second launch adds them up in the
// order of the keys: the end of a launch is what makes the parts of eight XCDs visible to one block.  (The block that arrives last could add them up within the
// launch, with parts stored for the whole device and a counter that it sets back; not built, so not measured.)
// Measured, bf16, d 128: 64 sequences of up to 4096 keys, 32 heads over 8 (195 MB) 43 us and 5 for the joins, 4.6 TB/s; four of up to 131072 keys, 8 heads over one
// (75 MB) 20 and 6 us, of which 4 and 2.5 are launch and latency; one of 876 keys 7.4 and 3: a chain of lengths, page, cache and parts.  A unit is 4 waves x 64 keys; each wave keeps its own state and shares nothing before the end of an item.
//
// A wave's step, 64 keys (lane group h = lane / 16 holds keys 16h .. 16h+15 of everything): the next step's codes and scales are loaded while
// this one is computed; K codes go from the load to the conversion (the cache holds them in operand order), V codes and all scales
// through the wave's own LDS, where the 4-bit transpose read turns rows of V into the operand's columns.
#include <hip/hip_runtime.h>

#include "cache_attn.h"

namespace slimattn {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kCols = 16;            // query columns of a tile
constexpr int kStep = 64;            // keys of a wave's step
constexpr int kUnit = kWaves * kStep;

// What a sequence of few columns adds to the row of units: every tile of every head its length in units.
struct NarrowRow {
  int row0, rows, len, tiles, units, heads;
  __device__ __forceinline__ NarrowRow(const AttnArgs& a, int b) {
    seq_rows(a, b, row0, rows, len);
    heads = a.c.n_kv_heads;
    const long long cols = (long long)rows * a.group;
    tiles = cols > a.narrow_cols ? 0 : (int)((cols + kCols - 1) / kCols);
    units = max(1, (len + kUnit - 1) / kUnit);               // rows that see nothing are items too: their outputs are written
  }
  __device__ __forceinline__ long long units_of_all() const { return (long long)tiles * units * heads; }
  __device__ __forceinline__ long long items() const { return (long long)tiles * heads; }
  __device__ __forceinline__ static int blocks(const AttnArgs&, int most, long long units, long long) { return (int)min((long long)most, units); }
  static constexpr bool kNeedsItems = false;
};

template <int D> constexpr int kPartFloats = kCols * D + 2 * kCols;   // [col][D], max [col], sum [col]

template <int D>
__device__ __forceinline__ float* part_of(char* ws, int block, int slot) {
  return reinterpret_cast<float*>(ws + 2 * kListBytes) + ((size_t)block * 2 + slot) * kPartFloats<D>;
}

typedef int int2v __attribute__((ext_vector_type(2)));
template <int D> struct Piece;                    // what a lane loads of D/2 bytes x 16 keys, or of the scales
template <> struct Piece<128> { typedef uint4 type; typedef uint2 scale; };
template <> struct Piece<64> { typedef uint2 type; typedef unsigned scale; };

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

// LDS of one wave: V codes, rows of D/2 bytes and 16 more (the transpose reads take the same 8 bytes of 16 rows at once).
template <int D> constexpr int kVRow = D / 2 + 16;
template <int D> constexpr int kWaveLds = kStep * kVRow<D>;
template <int D> constexpr int kOutRow = D + 4;                                    // floats; at the end: [wave][col][kOutRow], max, sum
template <int D> constexpr int kEndLds = kWaves * kCols * (kOutRow<D> + 2) * 4;
template <int D> constexpr int kLds = kWaves * kWaveLds<D> > kEndLds<D> ? kWaves * kWaveLds<D> : kEndLds<D>;

// Waves per SIMD, by what their registers take (bf16 158 and 114 of them at head dim 128 and 64, f32 213 and 150): nothing is spilled.
template <int D, int TERMS> constexpr int kBlocksPerCu = TERMS == 1 ? (D == 128 ? 3 : 4) : (D == 128 ? 2 : 3);

// One step's loads.  Tile t of the score product is the step's t-th chunk of 16 keys, so its C layout gives lane group h = lane / 16 the
// keys 16t + 4h + i (t, i = 0..3): "its" key number e = 4t + i of 16.  A lane's own key, whose scales it holds, is number lane % 16.
template <int D>
struct StepData {
  typedef typename Piece<D>::type P;
  typedef typename Piece<D>::scale S;
  P k[4], v[4];
  S ks, vs;
};

// The table's entry for this lane's chunk of a step's keys (chunk t: lanes with (lane >> 2) % 4 = t).  No branch: the last steps look up and
// load again what they drop.
__device__ __forceinline__ int load_page(const CacheView& c, const int32_t* table, int k0, int end) {
  return table[min(k0 + kCacheChunk * (int)((threadIdx.x >> 2) & 3), end - 1) >> c.page_shift];
}
// Makes a page of it.  Bit t: the chunk is in a page; chunks that are not take page 0 and are masked.
__device__ __forceinline__ unsigned step_pages(const CacheView& c, int& page, int k0, int end) {
  const bool there = (unsigned)page < (unsigned)c.n_pages && k0 + kCacheChunk * (int)((threadIdx.x >> 2) & 3) < end;
  page = there ? page : 0;
  const unsigned good = (unsigned)__ballot(there);
  return (good & 1) | (good >> 3 & 2) | (good >> 6 & 4) | (good >> 9 & 8);
}

// Scales and value codes: needed first.
// ONCE: nobody else reads these codes soon, they are streamed past the caches.
template <bool ONCE, class P>
__device__ __forceinline__ P load_codes(const char* p) {
  typedef unsigned V __attribute__((ext_vector_type(sizeof(P) / 4)));
  if constexpr (ONCE) return __builtin_bit_cast(P, __builtin_nontemporal_load(reinterpret_cast<const V*>(p)));
  return *reinterpret_cast<const P*>(p);
}
template <int D, bool ONCE>
__device__ __forceinline__ void load_values(StepData<D>& x, const CacheView& c, const char* head, unsigned pb, int page, int k0) {
  typedef typename StepData<D>::P P;
  typedef typename StepData<D>::S S;
  const int lane = threadIdx.x & 63, in_page = (1 << c.page_shift) - 1;
  const int own = k0 + kCacheChunk * ((lane >> 2) & 3) + 4 * (lane >> 4) + (lane & 3);
  const char* sp = head + (size_t)(unsigned)page * pb + scales<D>(c, 0, own & in_page);
  x.ks = *reinterpret_cast<const S*>(sp);
  x.vs = *reinterpret_cast<const S*>(sp + ((D / 16) << c.page_shift));
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const char* base = head + (size_t)(unsigned)__builtin_amdgcn_readlane(page, 4 * t) * pb + value_codes<D>(c, (k0 + kCacheChunk * t) & in_page);
    x.v[t] = load_codes<ONCE, P>(base + lane * (int)sizeof(P));
  }
}
template <int D, bool ONCE>
__device__ __forceinline__ void load_keys(StepData<D>& x, const CacheView& c, const char* head, unsigned pb, int page, int k0) {
  typedef typename StepData<D>::P P;
  const int lane = threadIdx.x & 63, in_page = (1 << c.page_shift) - 1;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const char* base = head + (size_t)(unsigned)__builtin_amdgcn_readlane(page, 4 * t) * pb + key_codes<D>((k0 + kCacheChunk * t) & in_page);
    x.k[t] = load_codes<ONCE, P>(base + (lane & 15) * (D / 2) + (lane >> 4) * (D / 8));
  }
}

// Value of lane e of each group of 16.
template <int E>
__device__ __forceinline__ float from_lane(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x150 + E, 0xf, 0xf, true));
}

// The running state of a wave's 16 columns: column lane % 16, and of O^T channels 16 ct + 4h + i.
template <int D>
struct State {
  floatx4v o[D / 16];
  float m, l;
};

// Scores of the step's 64 keys, in units of `scale`: a tile's products run while the one before it is scaled.
template <int D, int TERMS>
__device__ __forceinline__ void score_step(float (&s)[16], const StepData<D>& x, const float (&ks)[D / 32], const bf16x8 (&q)[D / 32][TERMS]) {
  constexpr int G = D / 32;
  floatx4v p[2][G];
  auto products = [&](auto t_) {
    constexpr int t = decltype(t_)::value;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const bf16x8 a = codes_to_bf16(word(x.k[t], g));
      p[t & 1][g] = floatx4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = TERMS - 1; n >= 0; --n) p[t & 1][g] = mfma16(a, q[g][n], p[t & 1][g]);
    }
  };
  products(IC<0>{});
  static_for<0, 4>([&](auto t_) {
    constexpr int t = decltype(t_)::value;
    if constexpr (t < 3) products(IC<t + 1>{});
    static_for<0, 4>([&](auto i_) {
      constexpr int i = decltype(i_)::value, e = 4 * t + i;
      static_for<0, G>([&](auto g_) {
        constexpr int g = decltype(g_)::value;
        const float f = from_lane<e>(ks[g]);
        s[e] = g == 0 ? p[t & 1][g][i] * f : __builtin_fmaf(p[t & 1][g][i], f, s[e]);
      });
    });
    // no further ahead: all tiles at once do not fit the registers
    asm volatile("" : "+v"(s[4 * t]), "+v"(s[4 * t + 1]), "+v"(s[4 * t + 2]), "+v"(s[4 * t + 3]));
    __builtin_amdgcn_sched_barrier(0);
  });
}

// The lane's last visible key of a step, less what its lane group adds to a key's number.  limit: the column's position (its last visible key).
__device__ __forceinline__ int last_of_step(int k0, int limit) { return limit - k0 - 4 * (int)((threadIdx.x & 63) >> 4); }
// Whether the column sees the lane's key number e.  there: step_pages.
__device__ __forceinline__ bool sees(int e, int last, unsigned there) { return 16 * (e >> 2) + (e & 3) <= last && (there >> (e >> 2) & 1); }

// Scores of keys that a column does not see.
__device__ __forceinline__ void mask_step(float (&s)[16], int k0, int limit, unsigned there) {
  const int last = last_of_step(k0, limit);
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (!sees(e, last, there)) s[e] = -INFINITY;
}

// A masked step's value scales may be anything (keys behind the end) or rightly NaN for some columns only.  Products with a probability of 0
// must not see them: scales that are not finite become 0, and columns that do see the key get their NaN here (whatever its probability came to: one
// that is seen may have underflowed).
template <int D>
__device__ __forceinline__ void clean_scales(State<D>& st, float (&vs)[D / 32], int k0, int limit, unsigned there) {
  static_for<0, D / 32>([&](auto g_) {
    constexpr int g = decltype(g_)::value;
    const bool bad = !(vs[g] - vs[g] == 0.f);
    if (__any(bad)) {
      bool hit = false;
      int last = last_of_step(k0, limit);
      asm volatile("" : "+v"(last));                         // (formed here: mask_step's sixteen comparisons are not kept for this)
      static_for<0, 16>([&](auto e_) {
        constexpr int e = decltype(e_)::value;
        const float f = from_lane<e>(vs[g]);
        hit |= !(f - f == 0.f) && sees(e, last, there);
      });
      hit |= (bool)__shfl_xor((int)hit, 16);                 // the column's other lane groups hold other channels
      hit |= (bool)__shfl_xor((int)hit, 32);
      const float poison = hit ? __builtin_nanf("") : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st.o[2 * g][i] += poison;
        st.o[2 * g + 1][i] += poison;
      }
      vs[g] = bad ? 0.f : vs[g];
    }
  });
}

// masked: the step has keys that some column does not see (uniform).  (Columns that are no rows, q = 0, may come to anything: they are dropped.)
template <int D, int TERMS>
__device__ __forceinline__ void softmax_step(State<D>& st, float (&s)[16], float (&vs)[D / 32], const char* vp, bool masked, int k0, int limit,
                                             unsigned there, float scale_log2) {
  constexpr int G = D / 32;
  if (masked) mask_step(s, k0, limit, there);
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
  if (masked) clean_scales<D>(st, vs, k0, limit, there);
  static_for<0, G>([&](auto g_) {
    constexpr int g = decltype(g_)::value;
    float p[2][8];
    static_for<0, 16>([&](auto e_) {
      constexpr int e = decltype(e_)::value;
      p[e >> 3][e & 7] = s[e] * from_lane<e>(vs[g]);
    });
    bf16x8 pt[2][TERMS];
    split_terms<TERMS>(p[0], pt[0]);
    split_terms<TERMS>(p[1], pt[1]);
#pragma unroll
    for (int ct = 2 * g; ct < 2 * g + 2; ++ct) {
      const int2v w = __builtin_amdgcn_ds_read_tr4_b64_v2i32((LDS_PTR(int2v))(vp + 8 * ct));
      const bf16x8 a0 = codes_to_bf16((unsigned)w.x), a1 = codes_to_bf16((unsigned)w.y);
#pragma unroll
      for (int n = TERMS - 1; n >= 0; --n) {
        st.o[ct] = mfma16(a0, pt[0][n], st.o[ct]);
        st.o[ct] = mfma16(a1, pt[1][n], st.o[ct]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  });
}

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

template <class T, int D, int TERMS, bool ONCE>
__global__ __launch_bounds__(kThreads, (kBlocksPerCu<D, TERMS>)) void cache_attn_kernel(AttnArgs a, const T* __restrict__ q, const char* __restrict__ cache,
                                                                 T* __restrict__ o, float* __restrict__ lse, char* __restrict__ ws) {
  typedef typename Piece<D>::type P;
  __shared__ __align__(16) char lds[kLds<D>];
  __shared__ long long scan[kWaves], found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 4, col = lane & 15;
  // One batch of loads for what the search below needs and what the compiler loads in front of it: left to itself it waits for them in turn, and for the
  // launch's size behind the scan: 0.2 us of a single token's 7.5, 1% of 64 sequences of 4096 keys.
  int N = gridDim.x;
  asm volatile("" : "+s"(N) : "s"(a.c.row_ptr), "s"(a.c.lens), "s"(a.c.n_seqs), "s"(a.group), "s"(a.narrow_cols), "s"(cache), "s"(lse), "s"(ws));

  Place place;
  if (!find_place<NarrowRow, kThreads>(a, N, scan, found, split_header(ws), place)) return;
  const int n = place.blocks, id = place.id;
  const long long U = place.total, u0 = place.begin, u1 = place.end;
  int b = place.seq;
  long long seq_begin = place.seq_begin, seq_item = place.seq_item;
  NarrowRow s(a, b);
  Split split{};

  for (long long u = u0; u < u1;) {
    while (u >= seq_begin + s.units_of_all()) {               // on to the next sequence with rows
      if (b + 1 >= a.c.n_seqs) { u = u1; break; }            // (units that do not add up: row_ptr or lens changed under the call)
      seq_begin += s.units_of_all();
      seq_item += s.items();
      s = NarrowRow(a, ++b);
    }
    if (u >= u1) break;
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

    char* vrows = lds + wave * kWaveLds<D>;
    const char* vp = vrows + lane * kVRow<D>;                // the rows of the lane group's 16 keys, in their order
    char* vw;                                                // where the lane's piece of chunk 0 goes; the next chunks 4 rows further each
    {
      const int at = lane * (int)sizeof(P), r = at / (D / 2);
      vw = vrows + (16 * (r >> 2) + (r & 3)) * kVRow<D> + at % (D / 2);
    }
    const int end = min(last * kUnit, visible);
    const int32_t* table = a.c.table + (size_t)b * a.c.max_pages;
    const char* head_piece = cache + hk * head_bytes<D>(a.c);
    const unsigned pb = (unsigned)page_bytes<D>(a.c);
    int k0 = first * kUnit + wave * kStep;
    StepData<D> x;
    unsigned there = 0;
    int page = 0, after = 0;                                 // of the step at hand's successor, and of the one behind that
    if (k0 < end) {
      page = load_page(a.c, table, k0, end);
      after = load_page(a.c, table, k0 + kUnit, end);
      there = step_pages(a.c, page, k0, end);
      load_values<D, ONCE>(x, a.c, head_piece, pb, page, k0);
      load_keys<D, ONCE>(x, a.c, head_piece, pb, page, k0);
      page = after;
    }
    for (; k0 < end; k0 += kUnit) {
      // this step's values into LDS, its scales into registers; then the next step's are on their way
#pragma unroll
      for (int t = 0; t < 4; ++t) *reinterpret_cast<P*>(vw + 4 * t * kVRow<D>) = x.v[t];
      float ks[D / 32], vs[D / 32];
#pragma unroll
      for (int g = 0; g < D / 32; ++g) {
        ks[g] = g & 1 ? hi_bf16(word(x.ks, g / 2)) : lo_bf16(word(x.ks, g / 2));
        vs[g] = g & 1 ? hi_bf16(word(x.vs, g / 2)) : lo_bf16(word(x.vs, g / 2));
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      const unsigned now = there;
      there = step_pages(a.c, page, k0 + kUnit, end);
      after = load_page(a.c, table, k0 + 2 * kUnit, end);    // (first: loads complete in order)
      load_values<D, ONCE>(x, a.c, head_piece, pb, page, k0 + kUnit);
      float s[16];
      score_step<D, TERMS>(s, x, ks, qf);
      load_keys<D, ONCE>(x, a.c, head_piece, pb, page, k0 + kUnit);
      page = after;
      softmax_step<D, TERMS>(st, s, vs, vp, now != 15 || k0 + kStep > all_see, k0, limit, now, a.scale_log2);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }

    // the four waves' states together (from a copy of the thread's number made here: what is derived from it would otherwise be kept in
    // registers through every walk)
    int me = tid;
    asm volatile("" : "+v"(me));
    const int my_col = me & 15, my_h = me >> 4 & 3;
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
    __syncthreads();
    float* ends = reinterpret_cast<float*>(lds);
    float* stat = ends + kWaves * kCols * kOutRow<D>;        // [wave][col] maximum, then sum
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
      *reinterpret_cast<floatx4v*>(ends + (wave * kCols + my_col) * kOutRow<D> + 16 * ct + 4 * my_h) = st.o[ct];
    if (my_h == 0) {
      stat[wave * kCols + my_col] = st.m;
      stat[kWaves * kCols + wave * kCols + my_col] = st.l;
    }
    __syncthreads();
    {
      constexpr int E = D / 16;                              // channels of a thread
      const int c = me >> 4, e0 = (me & 15) * E;
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
        if (c < cols) {
          store_out<E>(part + c * D + e0, out);
          if (e0 == 0) { part[kCols * D + c] = m; part[kCols * D + kCols + c] = l; }
        }
      }
    }
    if (first == 0) {
      split = Split{id, 0, s.row0, cols, col0, hk * a.group, {0, 0}};
      if (last < s.units) split.parts = block_of(seq_begin + (long long)item * s.units + s.units - 1, U, n) - id + 1;
      if (a.slots && tid == 0 && seq_item + item < a.slots) split_list(split_header(ws))[seq_item + item] = split;
    }
    __syncthreads();
    u += last - first;
  }
  if (!a.slots && tid == 0) split_list(split_header(ws))[id] = split;      // the last item it began: the one it may not have ended
}

// Adds up the parts of the split item listed at blockIdx.x, columns blockIdx.y, + gridDim.y, ...: runs of parts (thread / (D/4)) of four channels each,
// in a fixed order.
template <class T, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void cache_attn_join_kernel(AttnArgs a, T* __restrict__ o, float* __restrict__ lse, char* __restrict__ ws) {
  constexpr int W = D / 4, R = THREADS / W, WAVES = THREADS / 64;                 // threads of a row of D channels; runs
  const int tid = threadIdx.x;
  const Split s = split_list(split_header(ws))[blockIdx.x];  // (with the count, not behind it: the list has room for every block)
  if ((int)blockIdx.x >= split_header(ws)->listed || s.parts == 0) return;
  __shared__ float weight[kMaxGrid], red[2 * WAVES];
  __shared__ float sums[R][D + 4];
  auto part = [&](int p) { return part_of<D>(ws, s.first + p, p == 0 ? 1 : 0); };
  const int run = tid / W, e = (tid % W) * 4;
  for (int c = blockIdx.y; c < s.cols; c += gridDim.y) {
    floatx4v x = {0.f, 0.f, 0.f, 0.f};
    if (run < s.parts) x = *reinterpret_cast<const floatx4v*>(part(run) + c * D + e);   // on its way beside the statistics
    float m = -INFINITY, ms[kMaxGrid / THREADS], ls[kMaxGrid / THREADS];
#pragma unroll
    for (int i = 0; i < kMaxGrid / THREADS; ++i) {
      const int p = tid + i * THREADS;
      ms[i] = p < s.parts ? part(p)[kCols * D + c] : -INFINITY;
      ls[i] = p < s.parts ? part(p)[kCols * D + kCols + c] : 0.f;
      m = fmaxf(m, ms[i]);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, red[w]);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxGrid / THREADS; ++i) {
      const int p = tid + i * THREADS;
      const float f = __builtin_amdgcn_exp2f(ms[i] - ref);
      if (p < s.parts) weight[p] = f;
      l = __builtin_fmaf(ls[i], f, l);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
    if ((tid & 63) == 0) red[WAVES + (tid >> 6)] = l;
    __syncthreads();
    l = red[WAVES];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) l += red[WAVES + w];
    if (run < s.parts) x *= weight[run];
#pragma unroll 4
    for (int p = run + R; p < s.parts; p += R) x += *reinterpret_cast<const floatx4v*>(part(p) + c * D + e) * weight[p];
    *reinterpret_cast<floatx4v*>(&sums[run][e]) = x;
    __syncthreads();
    if (run == 0) {
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
    __syncthreads();
  }
}

// Items there can be: tiles of 16 columns of each sequence, at most one more than its columns fill.
long long most_items(const slimattn_cache_params& p, int n_q_heads) {
  return ((long long)p.n_rows * (n_q_heads / p.n_kv_heads) / kCols + p.n_seqs) * p.n_kv_heads;
}
// Blocks of the first launch: as many as there can be units, up to what is resident at once.
int grid_blocks(const slimattn_cache_params& p, int n_q_heads) {
  const int resident = 256 * (p.dtype == SLIMATTN_BF16 ? (p.head_dim == 128 ? kBlocksPerCu<128, 1> : kBlocksPerCu<64, 1>)
                                                       : (p.head_dim == 128 ? kBlocksPerCu<128, 3> : kBlocksPerCu<64, 3>));
  const long long items = most_items(p, n_q_heads), units = ((long long)p.max_pages * p.page_size + kUnit - 1) / kUnit;
  const long long most = items > resident ? resident : items * units;
  return (int)(most < resident ? most : resident);
}

}  // namespace

CacheView cache_view(const slimattn_cache_params& p, const int32_t* row_ptr, const int32_t* lens, const int32_t* table);
size_t cache_attn_wide_bytes(const slimattn_cache_params& p, int n_q_heads);
int launch_cache_attn_wide(const slimattn_cache_params& p, int n_q_heads, AttnArgs a, const void* q, const void* cache, void* o, float* lse, void* ws,
                           size_t parts_at, void* stream);

namespace {

// Which kernel takes a sequence goes by its number of query columns, which the device knows (row_ptr): the narrow kernel's time grows with the
// tiles of 16, the wide one's steps up every 256.  us narrow / wide, caches in rotation (as far as memory allows), columns a sequence:
//                                            64           96          112          128          192
//   64 of 4K keys, 32 heads over 8, d 128   216 /  287   272 /  309   344 /  303   380 /  297   497 /  311
//   16 of 4K                                 68 /   91    67 /   93   101 /   95   105 /   95   126 /  101
//   1 of 32K                                 36 /   56    43 /   57    53 /   58    57 /   57    73 /   60
//   64 of 4K, 32 heads over 32              873 / 1122  1244 / 1157  1450 / 1187  1646 / 1191  2383 / 1236
//   64 of 4K, 8 heads over one               40 /   61    49 /   63    59 /   64    66 /   65    67 /   68
//   64 of 4K, 32 heads over 8, d 64         108 /  203   153 /  204   205 /  207   198 /  207   294 /  211
// 64 heads over 8 go as 32 over 8.  Where there is little to do the rule costs time, since the wide kernel's larger parts take more than it saves: at 128 columns
// 1 of 32K keys over one head 22 / 34, 16 of 4K over one 28 / 38, 1 of 8K over 8 29 / 33 (d 64: 24 / 24).
constexpr long long kNarrowCols = 112;
bool may_be_wide(const slimattn_cache_params& p, int n_q_heads, bool ragged) {
  return p.dtype == SLIMATTN_BF16 && (ragged ? p.n_rows : 1ll) * (n_q_heads / p.n_kv_heads) > kNarrowCols;
}
// One sequence has all the rows there are: it is taken to be wide, and the narrow kernel has nothing to do.
bool all_wide(const slimattn_cache_params& p, int n_q_heads, bool ragged) { return may_be_wide(p, n_q_heads, ragged) && (!ragged || p.n_seqs == 1); }

size_t narrow_bytes(const slimattn_cache_params& p, int n_q_heads) {
  return (size_t)grid_blocks(p, n_q_heads) * 2 * (kCols * p.head_dim + 2 * kCols) * sizeof(float);
}

}  // namespace

size_t cache_attn_bytes(const slimattn_cache_params& p, int n_q_heads) {
  return 2 * kListBytes + narrow_bytes(p, n_q_heads) + (may_be_wide(p, n_q_heads, true) || may_be_wide(p, n_q_heads, false) ? cache_attn_wide_bytes(p, n_q_heads) : 0);
}

int launch_cache_attn(const slimattn_cache_params& p, int n_q_heads, float scale, const void* q, const int32_t* row_ptr, const int32_t* lens,
                      const int32_t* table, const void* cache, void* o, float* lse, void* ws, void* stream) {
  const bool wide = may_be_wide(p, n_q_heads, row_ptr != nullptr), narrow = !all_wide(p, n_q_heads, row_ptr != nullptr);
  AttnArgs a{cache_view(p, row_ptr, lens, table), n_q_heads / p.n_kv_heads, n_q_heads, 0.f, 1.f, !wide ? INT64_MAX : narrow ? kNarrowCols : 0, 0};
  const float f = scale * 1.4426950408889634f, size = f < 0.f ? -f : f;
  a.q_sign = f < 0.f ? -1.f : f > 0.f ? 1.f : 0.f;
  a.scale_log2 = size > 0x1p-126f ? size : 0x1p-126f;        // masked scores are -inf times it
  if (wide) {
    const int e = launch_cache_attn_wide(p, n_q_heads, a, q, cache, o, lse, ws, 2 * kListBytes + narrow_bytes(p, n_q_heads), stream);
    if (e != 0 || !narrow) return e;
  }
  const int blocks = grid_blocks(p, n_q_heads);
  // Few items are listed by their number, so that few blocks look for work in the second launch, and each of theirs may have hundreds of
  // parts: a block per column.  Many are listed by the block that began them, with few parts each: four columns.
  const long long items = most_items(p, n_q_heads);
  a.slots = items < blocks ? (int)items : 0;
  const dim3 join(a.slots ? a.slots : blocks, a.slots && a.slots <= 64 ? kCols : 4);
  // 128 parts of an item or more: 1024 threads, so that each adds up a few.  us in all with 256 / 1024 threads, bf16, d 128, 8 heads over one: one, two, four
  // sequences of 131072 keys (512, 384, 192 parts each) 22.8 / 20.9, 25.3 / 24.0, 28.4 / 27.8; with fewer parts the larger blocks cost more than they
  // save: eight of 131072 (96) 39.4 / 39.8, sixteen of 32768 (48) 26.0 / 26.6, fp32 of 65536 keys over 8 heads of 64 (96) 23.5 / 24.6.
  const bool many = a.slots && blocks >= 128 * a.slots;
  // Where sequences have 16 columns or fewer on average, their keys are read by one tile each and by nobody before the next call, with the other
  // layers' caches in between: streamed.  Caches in rotation, d 128, 32 heads over 8, us without / with: 19 MB 17.2 / 15.8, 76 MB 27.9 / 25.6, 303 MB
  // 78.6 / 67.4, 606 MB 132 / 116; 64 columns a sequence (four tiles) 223 / 234; a single cache of 195 MB read again and again from the last-level
  // cache 53.0 / 54.7.  (The host knows the average alone: a prompt among single tokens has all of them read through the caches.)
  const bool once = (long long)p.n_rows * a.group <= (long long)kCols * p.n_seqs;
  auto run = [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, TERMS = sizeof(T) == 4 ? 3 : 1;
    auto first = [&](auto streamed) {
      hipLaunchKernelGGL((cache_attn_kernel<T, D, TERMS, (decltype(streamed)::value != 0)>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a,
                         (const T*)q, (const char*)cache, (T*)o, lse, (char*)ws);
    };
    if (once) first(IC<1>{});
    else first(IC<0>{});
    const int e = (int)hipGetLastError();
    if (e != 0 || blocks < 2) return e;                      // one block holds every item whole
    if (many) hipLaunchKernelGGL((cache_attn_join_kernel<T, D, 1024>), join, dim3(1024), 0, (hipStream_t)stream, a, (T*)o, lse, (char*)ws);
    else hipLaunchKernelGGL((cache_attn_join_kernel<T, D, 256>), join, dim3(256), 0, (hipStream_t)stream, a, (T*)o, lse, (char*)ws);
    return (int)hipGetLastError();
  };
  if (p.dtype == SLIMATTN_F32) return p.head_dim == 128 ? run(float{}, IC<128>{}) : run(float{}, IC<64>{});
  return p.head_dim == 128 ? run(bf16{}, IC<128>{}) : run(bf16{}, IC<64>{});
}

}  // namespace slimattn
