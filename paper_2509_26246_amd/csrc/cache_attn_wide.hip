// Attention over the 4-bit cache for sequences with many query columns (rows x heads of the group): slices of prompts, bf16.
//
// The narrow kernel (cache_attn.hip) unpacks the cache once for 16 columns and scales scores and probabilities; with many columns that is most of its
// time.  Here a block of four waves takes 128 columns, and unpacks each tile of 64 keys once for all of them into LDS, scales applied: every value of
// the cache is exactly a bf16 number, so S^T = K q and O^T += V^T P^T on 32x32x16 products lose nothing against the codes.  Each wave keeps 32
// columns (a lane holds one column's scores, so sums and maxima need one lane exchange), tiles are double-buffered, and the next tile's codes are loaded a
// tile ahead and unpacked between the two products of this one.
//
// Bound by the vector unit: per wave and tile 32 products of 32 cycles against 32 exponentials of 16, and about 130 instructions to unpack a quarter
// of the next tile; two blocks share a compute unit, so one's products run beside the other's softmax.
//
// Work.  A tile's columns see the keys up to their last row, so the tiles of one prompt differ in length: a tile weighs (keys before the rows + a fixed
// part) * group + its last column's number, which adds up to a closed form over tiles; weights are divided evenly among the blocks, cuts fall on
// whole tiles of keys.  Parts leave O, maximum and sum of 128 columns in the workspace (67 KB at head dim 128): blocks are only used as far as each has
// the work of 256 keys, or an item of its own.
#include <hip/hip_runtime.h>

#include "cache_attn.h"

namespace slimattn {
namespace {

constexpr int kCols = 256;           // query columns of a block: two groups of 32 per wave
constexpr int kKeys = 64;            // keys of a tile
constexpr int kFixedKeys = 192;      // what an item costs beside its keys (its queries, its output), in keys
constexpr int kLeastKeys = 256;      // work that is worth a block and its parts
constexpr float kLazySum = 4096.f;   // the reference moves where a lane's sum of 16 probabilities exceeds this (or is not a number)

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

template <int D> constexpr int kPartFloats = kCols * D + 2 * kCols;
template <int D>
__device__ __forceinline__ float* part_of(char* parts, int block, int slot) { return reinterpret_cast<float*>(parts) + ((size_t)block * 2 + slot) * kPartFloats<D>; }

// What a sequence of many columns adds to the row of work: tile t of a head weighs weight(t), tiles 0 .. t-1 before(t).
struct WideRow {
  int row0, rows, len, tiles, heads, group;
  long long a;
  __device__ __forceinline__ WideRow(const AttnArgs& x, int b) {
    seq_rows(x, b, row0, rows, len);
    heads = x.c.n_kv_heads;
    group = x.group;
    const long long cols = (long long)rows * group;
    tiles = cols > x.narrow_cols ? (int)((cols + kCols - 1) / kCols) : 0;
    a = (long long)(max(len - rows, 0) + kFixedKeys) * group;
  }
  __device__ __forceinline__ long long weight(long long t) const { return a + kCols * (t + 1); }
  __device__ __forceinline__ long long before(long long t) const { return t * a + kCols * (t * (t + 1) / 2); }
  __device__ __forceinline__ long long units_of_all() const { return before(tiles) * heads; }
  __device__ __forceinline__ long long items() const { return (long long)tiles * heads; }
  // The tile in which unit y of a head lies: the root of before(t) = y, corrected for its rounding.
  __device__ __forceinline__ int tile_of(long long y) const {
    const double p = (double)a + 0.5 * kCols;
    long long t = (long long)((__builtin_sqrt(p * p + 2.0 * kCols * (double)y) - p) / kCols);
    t = min(max(t, 0ll), (long long)tiles - 1);
    while (t > 0 && before(t) > y) --t;
    while (t + 1 < tiles && before(t + 1) <= y) ++t;
    return (int)t;
  }
  // Keys of the cut at `w` of an item's weight.
  __device__ __forceinline__ int keys_at(long long w) const { return (int)max(w / group - kFixedKeys, 0ll) & ~(kKeys - 1); }
  __device__ __forceinline__ static int blocks(const AttnArgs& x, int most, long long units, long long items) {
    return (int)min((long long)most, max(items, units / ((long long)kLeastKeys * x.group)));
  }
  static constexpr bool kNeedsItems = true;
};

// The thread's number, as something to compute with here and now: offsets derived from it would otherwise be kept in registers through the walk, which
// has none to spare.
__device__ __forceinline__ int thread_number() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

// This thread's piece of a tile on its way: row tid / 4 (a wave's rows are one chunk of 16 keys), piece tid % 4 of its codes, and the scales.
template <int D>
struct Stage {
  static constexpr int G = D / 32;
  unsigned k[G], v[G], ks[G / 2], vs;
  int there;                         // bit c: the tile's chunk c is in a page (uniform)
};

// entry: lanes l hold the table's entry for chunk l % 4.  Chunks without a page take page 0 and are masked.
template <int D>
__device__ __forceinline__ void load_stage(Stage<D>& x, const CacheView& c, const char* head, unsigned pb, int entry, int k0, int end) {
  constexpr int G = D / 32;
  const int tid = thread_number(), wave = __builtin_amdgcn_readfirstlane(tid >> 6), key = k0 + kCacheChunk * wave;
  const bool good = (unsigned)entry < (unsigned)c.n_pages && k0 + kCacheChunk * (tid & 3) < end;
  x.there = (int)(__ballot(good) & 15);
  const int page = x.there >> wave & 1 ? __builtin_amdgcn_readlane(entry, wave) : 0;
  const int t = (key & ((1 << c.page_shift) - 1)) + (tid >> 2 & 15), j = tid & 3;
  const char* base = head + (size_t)(unsigned)page * pb;
  const unsigned* kp = reinterpret_cast<const unsigned*>(base + key_codes<D>(t)) + j * G;
  const unsigned* vp = reinterpret_cast<const unsigned*>(base + value_codes<D>(c, t)) + j * G;
  const unsigned* sp = reinterpret_cast<const unsigned*>(base + scales<D>(c, 0, t));
  if constexpr (G == 4) {
    const uint4 a = *reinterpret_cast<const uint4*>(kp), b = *reinterpret_cast<const uint4*>(vp);
    const uint2 s = *reinterpret_cast<const uint2*>(sp);
    x.k[0] = a.x; x.k[1] = a.y; x.k[2] = a.z; x.k[3] = a.w;
    x.v[0] = b.x; x.v[1] = b.y; x.v[2] = b.z; x.v[3] = b.w;
    x.ks[0] = s.x; x.ks[1] = s.y;
  } else {
    const uint2 a = *reinterpret_cast<const uint2*>(kp), b = *reinterpret_cast<const uint2*>(vp);
    x.k[0] = a.x; x.k[1] = a.y;
    x.v[0] = b.x; x.v[1] = b.y;
    x.ks[0] = *sp;
  }
  x.vs = *reinterpret_cast<const unsigned short*>(base + scales<D>(c, 1, t) + 2 * (j * G / 4));
}
// The table's entry for chunk lane % 4 of a tile.
__device__ __forceinline__ int load_entry(const CacheView& c, const int32_t* table, int k0, int end) {
  return table[min(k0 + kCacheChunk * (thread_number() & 3), end - 1) >> c.page_shift];
}

// Four codes (half a word, `hi`) times their scale.
__device__ __forceinline__ bf16x4 unpack4(unsigned w, bool hi, float s) {
  typedef float float2v __attribute__((ext_vector_type(2)));
  const float2v a = hi ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0);
  const float2v b = hi ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
  return __builtin_convertvector((floatx4){a.x * s, a.y * s, b.x * s, b.y * s}, bf16x4);
}

// LDS: [buffer][K tile, V tile], then per buffer and wave whether its chunk of the tile has scales that are not finite, and which of a key's groups
// those are (bits 0 .. G-1 values, 8 keys).  Rows are padded (K fragments: 16 lanes, rows one behind the other, take 16 bytes each; V^T fragments: 16 lanes
// take 4 rows x 32 bytes), so that every fragment is one lane address and a constant.
template <int D> constexpr int kKRow = D * 2 + 16;
template <int D> constexpr int kVRow = D * 2 + 32;
template <int D> constexpr int kBuffer = kKeys * (kKRow<D> + kVRow<D>);
template <int D> constexpr int kBadAt = 2 * kBuffer<D>;
constexpr int kBadBytes = 16 + kKeys * 4;
template <int D> constexpr int kLdsBytes = kBadAt<D> + 2 * kBadBytes;

// Where this thread's pieces of a tile go in a buffer: its first K word (channels 8 j ..; word g 64 bytes further each) and its first V word
// (channels 8 j G ..; word i 16 bytes further each).
template <int D>
__device__ __forceinline__ int unpack_keys_at(int tid) { return (tid >> 2) * kKRow<D> + (tid & 3) * 16; }
template <int D>
__device__ __forceinline__ int unpack_values_at(int tid) { return kKeys * kKRow<D> + (tid >> 2) * kVRow<D> + (tid & 3) * (D / 32) * 16; }

// Makes the scales of this thread's piece fit for products.  Chunks without a page and keys from `end` on (behind the last that some column of the
// block sees) may hold anything: their scales become zeros, and the softmax masks them.  So do scales that are not finite, which only columns
// that see their key may notice: the bits of those (note_bad; the softmax makes NaN of them for those columns).
template <int D>
__device__ __forceinline__ int clean_scales(Stage<D>& x, int k0, int end) {
  constexpr int G = D / 32;
  const int tid = thread_number(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned seen = (x.there >> wave & 1) && k0 + (tid >> 2) < end ? 0xffffffffu : 0u;
  auto odd = [](unsigned w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };   // halves whose exponent is all ones
  x.vs &= seen;
  unsigned any = odd(x.vs);
#pragma unroll
  for (int i = 0; i < G / 2; ++i) {
    x.ks[i] &= seen;
    any |= odd(x.ks[i]);
  }
  int bad = 0;
  if (__builtin_expect(__any(any != 0), 0)) {
#pragma unroll
    for (int i = 0; i < G / 2; ++i) {
      const unsigned w = odd(x.ks[i]);
      bad |= w ? 256 : 0;
      x.ks[i] &= (w & 0x8000u ? 0u : 0xffffu) | (w >> 31 ? 0u : 0xffff0000u);
    }
    const bool v = odd(x.vs) != 0;
    bad |= v ? 1 << ((tid & 3) * G / 4) : 0;
    x.vs = v ? 0u : x.vs;
  }
  return bad;
}
// Half of word n (key words, then value words) of the piece: n = slot / 2.  `part` takes the first half to the second.
template <int D>
__device__ __forceinline__ void unpack_slot(const Stage<D>& x, LDS_PTR(char) keys, LDS_PTR(char) values, int slot, bf16x4& part) {
  constexpr int G = D / 32;
  const int n = slot >> 1;
  const float s = n >= G ? lo_bf16(x.vs) : n & 1 ? hi_bf16(x.ks[n / 2]) : lo_bf16(x.ks[n / 2]);
  const bf16x4 y = unpack4(n >= G ? x.v[n - G] : x.k[n], slot & 1, s);
  if (slot & 1) *(LDS_PTR(bf16x8))(n >= G ? values + (n - G) * 16 : keys + n * 64) = __builtin_shufflevector(part, y, 0, 1, 2, 3, 4, 5, 6, 7);
  else part = y;
}
// What is not finite in the wave's chunk.
template <int D>
__device__ __forceinline__ void note_bad(LDS_PTR(char) lds, int buf, int bad) {
  const int tid = thread_number();
  LDS_PTR(int) info = (LDS_PTR(int))(lds + kBadAt<D> + buf * kBadBytes);
  const bool any = __any(bad != 0);
  info[tid >> 6] = any;                                      // (the wave's lanes write the same)
  if (any) {
    bad |= __shfl_xor(bad, 1);
    bad |= __shfl_xor(bad, 2);
    if ((tid & 3) == 0) info[4 + (tid >> 2)] = bad;
  }
}
template <int D>
__device__ __forceinline__ void unpack_stage(Stage<D>& x, LDS_PTR(char) lds, int buf, LDS_PTR(char) keys, LDS_PTR(char) values, int k0, int end) {
  const int bad = clean_scales<D>(x, k0, end);
  bf16x4 part;
#pragma unroll
  for (int slot = 0; slot < D / 8; ++slot) unpack_slot<D>(x, keys, values, slot, part);
  note_bad<D>(lds, buf, bad);
}

// Fragment f, issued before at most N later LDS operations, has landed.
template <int N>
__device__ __forceinline__ void wait_frag(bf16x8& f) { asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(f) : "n"(N)); }
template <int N>
__device__ __forceinline__ void wait_frag(short4v& a, short4v& b) { asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "n"(N)); }

// acc += a b, the accumulator in the accumulation registers (there are no others left for it): from inline asm, whose results and operands the
// compiler does not time.  Results are read by later products on the same accumulator or behind rest(); b and acc are written well ahead, or in
// front of rest_writes().
__device__ __forceinline__ void mfma_acc(floatx16& acc, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
template <int N>
__device__ __forceinline__ void rest(floatx16 (&acc)[2][N]) {
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int db = 0; db < N; ++db) asm volatile("s_nop 15" : "+a"(acc[g][db]));
  asm volatile("s_nop 15\n\ts_nop 15");
}
template <int N>
__device__ __forceinline__ void rest_writes(floatx16 (&acc)[2][N]) {
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int db = 0; db < N; ++db) asm volatile("s_nop 7" : "+a"(acc[g][db]));
}

__device__ __forceinline__ bf16x8 join_frag(short4v a, short4v b) {
  typedef __attribute__((__vector_size__(8 * sizeof(short)))) short short8v;
  return __builtin_bit_cast(bf16x8, (short8v)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int D>
__global__ __launch_bounds__(kThreads, 1) void cache_attn_wide_kernel(AttnArgs a, const bf16* __restrict__ q, const char* __restrict__ cache, bf16* __restrict__ o,
                                                                      float* __restrict__ lse, char* __restrict__ ws, size_t parts_at) {
  constexpr int NKS = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(1024))) char smem[kLdsBytes<D>];
  __shared__ long long scan[kWaves], found[3];
  LDS_PTR(char) lds = (LDS_PTR(char))smem;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
  const int N = gridDim.x;
  const int id = N % 8 == 0 ? (int)(blockIdx.x % 8) * (N / 8) + blockIdx.x / 8 : blockIdx.x;   // neighbours in the row of work on one XCD
  Header* header = split_header(ws + kListBytes);
  Place place;
  if (!find_place<WideRow>(a, N, id, scan, found, header, place)) return;
  int b = place.seq;
  long long seq_begin = place.seq_begin, seq_item = place.seq_item;
  WideRow s(a, b);
  Split split{};

  for (long long u = place.begin; u < place.end;) {
    while (u >= seq_begin + s.units_of_all()) {              // on to the next sequence with tiles
      if (b + 1 >= a.c.n_seqs) { u = place.end; break; }     // (units that do not add up: row_ptr or lens changed under the call)
      seq_begin += s.units_of_all();
      seq_item += s.items();
      s = WideRow(a, ++b);
    }
    if (u >= place.end) break;
    const long long per_head = s.before(s.tiles), local = u - seq_begin, head_begin = local / per_head * per_head;
    const int hk = __builtin_amdgcn_readfirstlane((int)(local / per_head)), t = __builtin_amdgcn_readfirstlane(s.tile_of(local - head_begin));
    const long long item_begin = seq_begin + head_begin + s.before(t), from = u - item_begin, to = min(s.weight(t), from + (place.end - u));
    const bool first = from == 0, last = to == s.weight(t);
    const long long col0 = (long long)t * kCols;             // columns of a sequence: rows * group may pass 32 bits
    const int cols = (int)min((long long)s.rows * a.group - col0, (long long)kCols);
    const int base = s.len - s.rows, row_first = (int)(col0 / a.group), in_row = (int)(col0 % a.group);
    const int visible = base + row_first + (in_row + cols - 1) / a.group + 1;
    const int wave_all = base + row_first + (in_row + wave * 64) / a.group + 1;                 // keys that all of the wave's columns see
    const int k_begin = first ? 0 : __builtin_amdgcn_readfirstlane(s.keys_at(from));
    const int k_end = __builtin_amdgcn_readfirstlane(last ? visible : min(s.keys_at(to), visible));

    bf16x8 qf[2][NKS];
    int limit[2];                                            // last key that the lane's columns see
    float m[2], l[2];                                        // their references (log2 units), their sums against them
    floatx16 oacc[2][NDB];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int mine = wave * 64 + 32 * g + l32, row = row_first + (in_row + mine) / a.group, head = hk * a.group + (in_row + mine) % a.group;
      const bool real = mine < cols;
      const bf16* qp = q + ((size_t)(s.row0 + (real ? row : 0)) * a.Hq + (real ? head : 0)) * D + 8 * half;
      const unsigned flip = a.q_sign < 0.f ? 0x80008000u : 0u, keep = real && a.q_sign != 0.f ? 0xffffffffu : 0u;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        uint4 w = *reinterpret_cast<const uint4*>(qp + 16 * ks);
        w.x = (w.x ^ flip) & keep; w.y = (w.y ^ flip) & keep; w.z = (w.z ^ flip) & keep; w.w = (w.w ^ flip) & keep;
        qf[g][ks] = __builtin_bit_cast(bf16x8, w);
      }
      limit[g] = real ? base + row - 4 * half : -64;         // less what the lane's half adds to a key's number
      m[g] = real ? -INFINITY : 0.f;
      l[g] = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[g][db][r] = 0.f;
        asm volatile("" : "+a"(oacc[g][db]));
      }
    }
    rest_writes(oacc);

    const int32_t* table = a.c.table + (size_t)b * a.c.max_pages;
    const char* piece = cache + hk * head_bytes<D>(a.c);
    const unsigned pb = (unsigned)page_bytes<D>(a.c);
    if (k_begin < k_end) {
      // two tiles on their way beside the one at hand
      Stage<D> xa, xb;
      const int e0 = load_entry(a.c, table, k_begin, k_end), e1 = load_entry(a.c, table, k_begin + kKeys, k_end), e2 = load_entry(a.c, table, k_begin + 2 * kKeys, k_end);
      int entry = load_entry(a.c, table, k_begin + 3 * kKeys, k_end);
      load_stage<D>(xa, a.c, piece, pb, e0, k_begin, k_end);
      load_stage<D>(xb, a.c, piece, pb, e1, k_begin + kKeys, k_end);
      __syncthreads();                                       // the buffers are free
      unpack_stage<D>(xa, lds, 0, lds + unpack_keys_at<D>(tid), lds + unpack_values_at<D>(tid), k_begin, visible);
      int there = xa.there;
      load_stage<D>(xa, a.c, piece, pb, e2, k_begin + 2 * kKeys, k_end);
      __syncthreads();
      // this buffer's fragments, the other's unpacked pieces
      lds_cptr pk = keep(lds + l32 * kKRow<D> + 16 * half);
      lds_cptr pv = keep(lds + kKeys * kKRow<D> + (4 * (lane >> 5) + (lane >> 2 & 3)) * kVRow<D> + 32 * (lane >> 4 & 1) + 8 * (lane & 3));
      LDS_PTR(char) uk = lds + kBuffer<D> + unpack_keys_at<D>(tid);
      LDS_PTR(char) uv = lds + kBuffer<D> + unpack_values_at<D>(tid);

      // The products of tile k0 in buffer BUF, and between them the other work: x, the next tile, is unpacked beside the first half's scores and the
      // second half's O^T products; a half's probabilities are formed beside the products that follow its scores.  A half is 32 keys.  A
      // fragment serves both groups of columns; fragments are read kAhead ahead of their products.
      auto tile = [&](auto buf_, Stage<D>& x, const int k0) {
        constexpr int BUF = decltype(buf_)::value, NF = 2 * NKS, NV = 4 * NDB, kAhead = 3;
        const bool masked = there != 15 || k0 + kKeys > wave_all;
        auto mask = [&](floatx16& s, int kb, int g) {        // key 32 kb + 8 (r / 4) + 4 half + r % 4 of the tile
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kb + 8 * (r >> 2) + (r & 3) > limit[g] - k0 || !(there >> (2 * kb + (r >> 3)) & 1)) s[r] = -INFINITY;
        };
        floatx16 sacc[2][2];                                 // [half][group]
        bf16x8 kf[NF];
        short4v vf[NV][2];
        auto issue = [&](auto o_) {
          constexpr int o = decltype(o_)::value;
          if constexpr (o < NF) {
            r1_issue<(o / NKS) * 32 * kKRow<D> + (o % NKS) * 32>(pk, kf[o]);
          } else if constexpr (o < NF + NV) {
            constexpr int p = o - NF;
            tr1_issue<(p / NDB) * 16 * kVRow<D> + (p % NDB) * 64>(pv, vf[p][0]);
            tr1_issue<((p / NDB) * 16 + 8) * kVRow<D> + (p % NDB) * 64>(pv, vf[p][1]);
          }
        };
        constexpr auto later = [](int o) {                   // LDS reads issued behind fragment o's when it is used
          int n = 0;
          for (int i = o + 1; i < o + kAhead && i < NF + NV; ++i) n += i < NF ? 1 : 2;
          return n;
        };
        unsigned pf[2][2][8];
        float sum[2], y[2], ref[2];
        auto probability = [&](auto kb_, int g, const floatx16& s, int e) {
          constexpr int kb = decltype(kb_)::value;
          const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale_log2, -ref[g]));
          sum[g] = e == 0 ? z : sum[g] + z;
          if (e & 1) {
            typedef float float2v __attribute__((ext_vector_type(2)));
            unsigned w = __builtin_bit_cast(unsigned, __builtin_convertvector((float2v){y[g], z}, bf16x2v));
            asm volatile("" : "+v"(w));                      // (packed here: not the two floats kept)
            pf[kb][g][e >> 1] = w;
          }
          y[g] = z;
        };
        // A half's references: they move (rarely) where a lane's sum gets large, and from -inf at the first key that is seen; the half's scores and
        // probabilities are formed again.  (Scores kept for this case would cost registers in every tile.)
        auto settle = [&](auto kb_) {
          constexpr int kb = decltype(kb_)::value;
          const bool moves = !(fmaxf(sum[0], sum[1]) <= kLazySum) || sum[0] != sum[0] || sum[1] != sum[1] || fminf(m[0], m[1]) == -INFINITY;
          if (__builtin_expect(__any(moves), 0)) {
            rest(oacc);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              floatx16 s;
#pragma unroll
              for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
              for (int ks = 0; ks < NKS; ++ks)
                s = mfma32(*(LDS_PTR(const bf16x8))(pk + kb * 32 * kKRow<D> + ks * 32), qf[g][ks], s);
              if (masked) mask(s, kb, g);
              float mx = s[0];
#pragma unroll
              for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
              mx = fmaxf(mx, xor32(mx)) * a.scale_log2;
              const float to_m = fmaxf(m[g], mx), alpha = to_m == m[g] ? 1.f : __builtin_amdgcn_exp2f(m[g] - to_m);
              m[g] = to_m;
              l[g] *= alpha;
#pragma unroll
              for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[g][db][r] *= alpha;
              ref[g] = m[g] == -INFINITY ? 0.f : m[g];
#pragma unroll
              for (int e = 0; e < 16; ++e) probability(kb_, g, s, e);
            }
            rest_writes(oacc);
          }
          l[0] += sum[0];
          l[1] += sum[1];
        };
        auto weights = [&](int j, int g) {
          typedef unsigned uint4v __attribute__((ext_vector_type(4)));
          const unsigned* w = &pf[j >> 1][g][4 * (j & 1)];
          return __builtin_bit_cast(bf16x8, (uint4v){w[0], w[1], w[2], w[3]});
        };
        // a half's 32 probabilities beside products 2 .. 2 NKS - 1 (the scores are still on their way beside the first two)
        auto share = [&](auto kb_, auto i_) {
          constexpr int i = decltype(i_)::value, n = 2 * NKS - 2;
          if constexpr (i >= 2)
            static_for<(i - 2) * 32 / n, (i - 1) * 32 / n>([&](auto e_) {
              constexpr int e = decltype(e_)::value;
              probability(kb_, e & 1, sacc[decltype(kb_)::value][e & 1], e >> 1);
            });
        };
        const int bad = clean_scales<D>(x, k0 + kKeys, visible);
        bf16x4 part;
        static_for<0, kAhead>([&](auto o_) { issue(o_); });
        static_for<0, 2 * NKS>([&](auto i_) {
          constexpr int i = decltype(i_)::value, ks = i / 2, g = i % 2;
          if constexpr (g == 0) wait_frag<later(ks)>(kf[ks]);
          if constexpr (g == 0) unpack_slot<D>(x, uk, uv, ks, part);
          if constexpr (ks == 0) {
            const floatx16 zero = {};
            sacc[0][g] = mfma32(kf[ks], qf[g][ks], zero);
          } else {
            sacc[0][g] = mfma32(kf[ks], qf[g][ks], sacc[0][g]);
          }
          if constexpr (g == 1) issue(IC<ks + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        if (masked) {
          mask(sacc[0][0], 0, 0);
          mask(sacc[0][1], 0, 1);
        }
        ref[0] = m[0] == -INFINITY ? 0.f : m[0];
        ref[1] = m[1] == -INFINITY ? 0.f : m[1];
        static_for<0, 2 * NKS>([&](auto i_) {
          constexpr int i = decltype(i_)::value, ks = i / 2, g = i % 2, o = NKS + ks;
          if constexpr (g == 0) wait_frag<later(o)>(kf[o]);
          share(IC<0>{}, i_);
          if constexpr (ks == 0) {
            const floatx16 zero = {};
            sacc[1][g] = mfma32(kf[o], qf[g][ks], zero);
          } else {
            sacc[1][g] = mfma32(kf[o], qf[g][ks], sacc[1][g]);
          }
          if constexpr (g == 1) issue(IC<o + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        settle(IC<0>{});
        if (masked) {
          mask(sacc[1][0], 1, 0);
          mask(sacc[1][1], 1, 1);
        }
        asm volatile("s_nop 7");                             // the last probabilities are written: see mfma_acc
        static_for<0, 4 * NDB>([&](auto i_) {
          constexpr int i = decltype(i_)::value, p = i / 2, g = i % 2;
          if constexpr (g == 0) wait_frag<later(NF + p)>(vf[p][0], vf[p][1]);
          share(IC<1>{}, i_);
          mfma_acc(oacc[g][p % NDB], join_frag(vf[p][0], vf[p][1]), weights(p / NDB, g));
          if constexpr (g == 1) issue(IC<NF + p + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        settle(IC<1>{});
        LDS_PTR(const int) info = (LDS_PTR(const int))(lds + kBadAt<D> + BUF * kBadBytes);
        const int any_bad = info[0] | info[1] | info[2] | info[3];
        asm volatile("s_nop 7");
        static_for<0, 4 * NDB>([&](auto i_) {
          constexpr int i = decltype(i_)::value, p = 2 * NDB + i / 2, g = i % 2;
          if constexpr (g == 0) wait_frag<later(NF + p)>(vf[p][0], vf[p][1]);
          if constexpr (g == 0) unpack_slot<D>(x, uk, uv, NKS + i / 2, part);
          mfma_acc(oacc[g][p % NDB], join_frag(vf[p][0], vf[p][1]), weights(p / NDB, g));
          if constexpr (g == 1) issue(IC<NF + p + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        note_bad<D>(lds, BUF ^ 1, bad);
        if (__builtin_amdgcn_readfirstlane(any_bad)) {       // scales that are not finite: NaN where their keys are seen
          rest(oacc);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            int hit = 0;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int key = 32 * kb + 8 * (r >> 2) + (r & 3), chunk = 2 * kb + (r >> 3);
                hit |= info[chunk] && k0 + key <= limit[g] ? info[4 + key + 4 * half] : 0;
              }
            hit |= __shfl_xor(hit, 32);
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
              const float poison = hit & (256 | 1 << db) ? __builtin_nanf("") : 0.f;
#pragma unroll
              for (int r = 0; r < 16; ++r) oacc[g][db][r] += poison;
            }
            l[g] += hit & 256 ? __builtin_nanf("") : 0.f;
          }
          rest_writes(oacc);
        }
        there = x.there;
        const int entry_now = entry;
        entry = load_entry(a.c, table, k0 + 4 * kKeys, k_end);   // (first: loads complete in order)
        load_stage<D>(x, a.c, piece, pb, entry_now, k0 + 3 * kKeys, k_end);
        constexpr int to_other = BUF ? -kBuffer<D> : kBuffer<D>;
        pk += to_other; pv += to_other;
        uk -= to_other; uv -= to_other;
        // this tile's reads and the next one's writes are done (loads on their way may stay so)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      };
      // (Tiles in pairs, without a branch: an odd number's last partner has no chunk in a page and adds nothing, and the last tiles load and unpack
      // again what nobody reads.)
      for (int k0 = k_begin; k0 < k_end; k0 += 2 * kKeys) {
        tile(IC<0>{}, xb, k0);
        tile(IC<1>{}, xa, k0 + kKeys);
      }
    }
    rest(oacc);

    // (the columns again, from a copy of the thread's number: their places in the outputs would otherwise be kept in registers through the walk)
    const int me = thread_number(), out_half = me >> 5 & 1;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int col = (me >> 6) * 64 + 32 * g + (me & 31), row = row_first + (in_row + col) / a.group, head = hk * a.group + (in_row + col) % a.group;
      const float total = l[g] + xor32(l[g]);
      if (col >= cols) continue;
      if (first && last) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        bf16* op = o + ((size_t)(s.row0 + row) * a.Hq + head) * D + 4 * out_half;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = total == 0.f ? 0.f : oacc[g][db][r + e] * inv;
            store_out<4>(op + 32 * db + 2 * r, x);
          }
        if (lse && out_half == 0) lse[(size_t)head * a.c.n_rows + s.row0 + row] = (m[g] + __builtin_amdgcn_logf(total)) * kLn2;
      } else {
        float* part = part_of<D>(ws + parts_at, id, first ? 1 : 0);
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<floatx4v*>(part + col * D + 32 * db + 2 * r + 4 * out_half) = floatx4v{oacc[g][db][r], oacc[g][db][r + 1], oacc[g][db][r + 2], oacc[g][db][r + 3]};
        if (out_half == 0) { part[kCols * D + col] = m[g]; part[kCols * D + kCols + col] = total; }
      }
    }
    if (first) {
      const long long item_end = item_begin + s.weight(t);
      split = Split{id, 0, s.row0 + row_first, cols, in_row, hk * a.group, {0, 0}};
      if (!last) split.parts = block_of(item_end - 1, place.total, place.blocks) - id + 1;
      const long long number = seq_item + (long long)hk * s.tiles + t;
      if (a.slots && tid == 0 && number < a.slots) split_list(header)[number] = split;
    }
    u += to - from;
  }
  if (!a.slots && tid == 0) split_list(header)[id] = split;
}

// Adds up the parts of the split item listed at blockIdx.x, in order: a thread has four channels of one column.
template <int D>
__global__ __launch_bounds__(kThreads) void cache_attn_wide_join_kernel(AttnArgs a, bf16* __restrict__ o, float* __restrict__ lse, char* __restrict__ ws, size_t parts_at) {
  constexpr int W = D / 4;
  Header* header = split_header(ws + kListBytes);
  if ((int)blockIdx.x >= header->listed) return;
  const Split s = split_list(header)[blockIdx.x];
  const int c = blockIdx.y * (kThreads / W) + threadIdx.x / W, e = threadIdx.x % W * 4;
  if (s.parts == 0 || c >= s.cols) return;
  auto part = [&](int p) { return part_of<D>(ws + parts_at, s.first + p, p == 0 ? 1 : 0); };
  float m = -INFINITY;
#pragma unroll 8
  for (int p = 0; p < s.parts; ++p) m = fmaxf(m, part(p)[kCols * D + c]);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  floatx4v x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < s.parts; ++p) {
    const float* y = part(p);
    const float f = __builtin_amdgcn_exp2f(y[kCols * D + c] - ref);
    l = __builtin_fmaf(y[kCols * D + kCols + c], f, l);
    x += *reinterpret_cast<const floatx4v*>(y + c * D + e) * f;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int r = s.row0 + (s.col0 + c) / a.group, hd = s.head0 + (s.col0 + c) % a.group;
  const float out[4] = {l == 0.f ? 0.f : x[0] * inv, l == 0.f ? 0.f : x[1] * inv, l == 0.f ? 0.f : x[2] * inv, l == 0.f ? 0.f : x[3] * inv};
  store_out<4>(o + ((size_t)r * a.Hq + hd) * D + e, out);
  if (lse && e == 0) lse[(size_t)hd * a.c.n_rows + r] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

long long most_items(const slimattn_cache_params& p, int n_q_heads) {
  return ((long long)p.n_rows * (n_q_heads / p.n_kv_heads) / kCols + p.n_seqs) * p.n_kv_heads;
}
// A block per compute unit, fewer where there cannot be work for them.
int grid_blocks(const slimattn_cache_params& p, int n_q_heads) {
  const long long items = most_items(p, n_q_heads), keys = (long long)p.max_pages * p.page_size + kFixedKeys + 1;
  const long long most = items > 256 ? 256 : items * (keys / kLeastKeys + 1);
  return (int)(most < 256 ? most : 256);
}

}  // namespace

size_t cache_attn_wide_bytes(const slimattn_cache_params& p, int n_q_heads) {
  return (size_t)grid_blocks(p, n_q_heads) * 2 * (kCols * p.head_dim + 2 * kCols) * sizeof(float);
}

int launch_cache_attn_wide(const slimattn_cache_params& p, int n_q_heads, AttnArgs a, const void* q, const void* cache, void* o, float* lse, void* ws,
                           size_t parts_at, void* stream) {
  const int blocks = grid_blocks(p, n_q_heads);
  const long long items = most_items(p, n_q_heads);
  a.slots = items < blocks ? (int)items : 0;
  auto run = [&](auto d) {
    constexpr int D = decltype(d)::value;
    hipLaunchKernelGGL((cache_attn_wide_kernel<D>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const bf16*)q, (const char*)cache,
                       (bf16*)o, lse, (char*)ws, parts_at);
    const int e = (int)hipGetLastError();
    if (e != 0 || blocks < 2) return e;
    hipLaunchKernelGGL((cache_attn_wide_join_kernel<D>), dim3(a.slots ? a.slots : blocks, kCols * (D / 4) / kThreads), dim3(kThreads), 0, (hipStream_t)stream, a,
                       (bf16*)o, lse, (char*)ws, parts_at);
    return (int)hipGetLastError();
  };
  return p.head_dim == 128 ? run(IC<128>{}) : run(IC<64>{});
}

}  // namespace slimattn
