// Attention over the 4-bit cache for sequences with many query columns (rows x heads of the group): slices of prompts, bf16.
//
// The narrow kernel (cache_attn.hip) unpacks the cache once for 16 columns and scales scores and probabilities; with many columns that is most of its
// time.  Here a block of eight waves takes 256 columns, and unpacks each tile of 64 keys once for all of them into LDS, scales applied: every value of
// the cache is exactly a bf16 number, so S^T = K q and O^T += V^T P^T on 32x32x16 products lose nothing against the codes.  Each wave keeps 32
// columns (a lane holds one column's scores, so sums and maxima need one lane exchange), tiles are double-buffered, and the next tile's codes are loaded
// a tile ahead of that and unpacked beside the products of this one.  LDS rows are padded, so that a fragment is one address and a constant.
//
// Probabilities are rounded to bf16 for the second product, as slimattn_fwd rounds them (at most 2^-8 of each term; the sum takes them unrounded): a
// second term would make that product two, half as much again of all the matrix work, for an error of 1.65e-3 instead of 2.3e-3 (cache_attn.hip).
//
// 1024 new rows behind 31K keys, 8 heads over one, head dim 128 (135 GFLOP): 157 to 165 us in all, 820 to 860 TFLOP/s; the narrow kernel takes 293 us.  A tile of 64 keys
// takes a compute unit 2 us (1050 TFLOP/s; a large library product reaches 1220), the rest is fixed: finding the work, first loads, parts, join.  No
// single part binds a tile: matrix unit 43% of the cycles, vector unit 50%, LDS 45%; without the exponentials, the second product, the unpacking
// or the loads (each taken out alone) 5 to 8% go.  Within 4% of it came four waves of 32 columns, two blocks to a compute unit, and four waves of 64
// columns; within 1% four buffers with a barrier every second tile, V rows padded for half the reads' conflicts, and wave priorities.
//
// Work.  A tile's columns see the keys up to their last row, so the tiles of one prompt differ in length: a tile weighs (keys before the rows + a fixed
// part) * group + its last column's number, which adds up to a closed form over tiles; weights are divided evenly among the blocks, cuts fall on
// whole tiles of keys.  Parts leave O, maximum and sum of 256 columns in the workspace (133 KB at head dim 128): blocks are only used as far as each has
// the work of 256 keys, or an item of its own.
#include <hip/hip_runtime.h>

#include "cache_attn.h"

namespace slimattn {
namespace {

constexpr int kThreads = 512, kWaves = 8;
constexpr int kCols = 32 * kWaves;   // query columns of a block, 32 per wave
constexpr int kKeys = 64;            // keys of a tile
constexpr int kFixedKeys = 192;      // what an item costs beside its keys (its queries, its output), in keys
constexpr int kLeastKeys = 256;      // work that is worth a block and its parts
constexpr float kLazySum = 4096.f;   // the reference moves where a lane's sum of 16 probabilities exceeds this (or is not a number)

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// A part: O^T as the waves hold it, [wave][32 channels][8 channels][lane] of four floats, then maximum and sum of each column.
template <int D> constexpr int kPartFloats = kCols * D + 2 * kCols;
template <int D>
__device__ __forceinline__ int part_at(int wave, int db, int r4, int lane) { return (((wave * (D / 32) + db) * 4 + r4) * 64 + lane) * 4; }
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

// This thread's piece of a tile on its way: row tid / 8 (a wave's rows are half a chunk of 16 keys), piece tid % 8 of its codes, and the scales
// of its keys (two groups at head dim 128, one at 64) and values.
template <int D>
struct Stage {
  static constexpr int W = D / 64;   // words of a piece
  unsigned k[W], v[W], ks, vs;
  int there;                         // bit c: the tile's chunk c is in a page (uniform)
};

// entry: lanes l hold the table's entry for chunk l % 4.  Chunks without a page take page 0 and are masked.
template <int D>
__device__ __forceinline__ void load_stage(Stage<D>& x, const CacheView& c, const char* head, unsigned pb, int entry, int k0, int end) {
  const int tid = thread_number(), chunk = __builtin_amdgcn_readfirstlane(tid >> 7), key = k0 + kCacheChunk * chunk;
  const bool good = (unsigned)entry < (unsigned)c.n_pages && k0 + kCacheChunk * (tid & 3) < end;
  x.there = (int)(__ballot(good) & 15);
  const int page = x.there >> chunk & 1 ? __builtin_amdgcn_readlane(entry, chunk) : 0;
  const int t = (key & ((1 << c.page_shift) - 1)) + (tid >> 3 & 15), j = tid & 7;
  const char* base = head + (size_t)(unsigned)page * pb;
  const unsigned* kp = reinterpret_cast<const unsigned*>(base + key_codes<D>(t)) + j * Stage<D>::W;
  const unsigned* vp = reinterpret_cast<const unsigned*>(base + value_codes<D>(c, t)) + j * Stage<D>::W;
  const char* sp = base + scales<D>(c, 0, t);
  if constexpr (D == 128) {                                  // key words 2 j, 2 j + 1: lane group j / 2, scale groups 2 (j % 2) and the next
    const uint2 a = *reinterpret_cast<const uint2*>(kp), b = *reinterpret_cast<const uint2*>(vp);
    x.k[0] = a.x; x.k[1] = a.y;
    x.v[0] = b.x; x.v[1] = b.y;
    x.ks = *reinterpret_cast<const unsigned*>(sp + 4 * (j & 1));
  } else {                                                   // key word j: lane group j / 2, scale group j % 2
    x.k[0] = *kp;
    x.v[0] = *vp;
    x.ks = *reinterpret_cast<const unsigned short*>(sp + 2 * (j & 1));
  }
  x.vs = *reinterpret_cast<const unsigned short*>(base + scales<D>(c, 1, t) + 2 * (j * Stage<D>::W / 4));
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
constexpr int kBadBytes = 32 + kKeys * 4;
template <int D> constexpr int kLdsBytes = kBadAt<D> + 2 * kBadBytes;

// Where this thread's pieces of a tile go in a buffer: its first K word (the next one's channels lie 64 bytes further) and its first V word.
template <int D>
__device__ __forceinline__ int unpack_keys_at(int tid) {
  return (tid >> 3) * kKRow<D> + (tid & 1) * (D == 128 ? 128 : 64) + (tid >> 1 & 3) * 16;
}
template <int D>
__device__ __forceinline__ int unpack_values_at(int tid) { return kKeys * kKRow<D> + (tid >> 3) * kVRow<D> + (tid & 7) * (D / 64) * 16; }

// Makes the scales of this thread's piece fit for products.  Chunks without a page and keys from `end` on (behind the last that some column of the
// block sees) may hold anything: their scales become zeros, and the softmax masks them.  So do scales that are not finite, which only columns
// that see their key may notice: the bits of those (note_bad; the softmax makes NaN of them for those columns).
template <int D>
__device__ __forceinline__ int clean_scales(Stage<D>& x, int k0, int end) {
  const int tid = thread_number(), chunk = __builtin_amdgcn_readfirstlane(tid >> 7);
  const unsigned seen = (x.there >> chunk & 1) && k0 + (tid >> 3) < end ? 0xffffffffu : 0u;
  auto odd = [](unsigned w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };   // halves whose exponent is all ones
  x.vs &= seen;
  x.ks &= seen;
  int bad = 0;
  if (__builtin_expect(__any((odd(x.vs) | odd(x.ks)) != 0), 0)) {
    const unsigned w = odd(x.ks);
    bad |= w ? 256 : 0;
    x.ks &= (w & 0x8000u ? 0u : 0xffffu) | (w >> 31 ? 0u : 0xffff0000u);
    const bool v = odd(x.vs) != 0;
    bad |= v ? 1 << ((tid & 7) * (D / 64) / 4) : 0;
    x.vs = v ? 0u : x.vs;
  }
  return bad;
}
// Half of word n (key words, then value words) of the piece: n = slot / 2, slots 0 .. D/16 - 1.  `part` takes the first half to the second.
template <int D>
__device__ __forceinline__ void unpack_slot(const Stage<D>& x, LDS_PTR(char) keys, LDS_PTR(char) values, int slot, bf16x4& part) {
  constexpr int W = D / 64;
  const int n = slot >> 1;
  const float s = n >= W ? lo_bf16(x.vs) : n & 1 ? hi_bf16(x.ks) : lo_bf16(x.ks);
  const bf16x4 y = unpack4(n >= W ? x.v[n - W] : x.k[n], slot & 1, s);
  if (slot & 1) *(LDS_PTR(bf16x8))(n >= W ? values + (n - W) * 16 : keys + n * 64) = __builtin_shufflevector(part, y, 0, 1, 2, 3, 4, 5, 6, 7);
  else part = y;
}
// What is not finite in the wave's keys.
template <int D>
__device__ __forceinline__ void note_bad(LDS_PTR(char) lds, int buf, int bad) {
  const int tid = thread_number();
  LDS_PTR(int) info = (LDS_PTR(int))(lds + kBadAt<D> + buf * kBadBytes);
  const bool any = __any(bad != 0);
  info[tid >> 6] = any;                                      // (the wave's lanes write the same)
  if (any) {
    bad |= __shfl_xor(bad, 1);
    bad |= __shfl_xor(bad, 2);
    bad |= __shfl_xor(bad, 4);
    if ((tid & 7) == 0) info[kWaves + (tid >> 3)] = bad;
  }
}
template <int D>
__device__ __forceinline__ void unpack_stage(Stage<D>& x, LDS_PTR(char) lds, int buf, LDS_PTR(char) keys, LDS_PTR(char) values, int k0, int end) {
  const int bad = clean_scales<D>(x, k0, end);
  bf16x4 part;
#pragma unroll
  for (int slot = 0; slot < D / 16; ++slot) unpack_slot<D>(x, keys, values, slot, part);
  note_bad<D>(lds, buf, bad);
}

// Fragment f, issued before at most N later LDS operations, has landed.
template <int N>
__device__ __forceinline__ void wait_frag(bf16x8& f) { asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(f) : "n"(N)); }
template <int N>
__device__ __forceinline__ void wait_frag(short4v& a, short4v& b) { asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "n"(N)); }

__device__ __forceinline__ bf16x8 join_frag(short4v a, short4v b) {
  typedef __attribute__((__vector_size__(8 * sizeof(short)))) short short8v;
  return __builtin_bit_cast(bf16x8, (short8v)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_wide_kernel(AttnArgs a, const bf16* __restrict__ q, const char* __restrict__ cache, bf16* __restrict__ o,
                                                                      float* __restrict__ lse, char* __restrict__ ws, size_t parts_at) {
  constexpr int NKS = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(1024))) char smem[kLdsBytes<D>];
  __shared__ long long scan[kWaves], found[3];
  LDS_PTR(char) lds = (LDS_PTR(char))smem;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
  Header* header = split_header(ws + kListBytes);
  Place place;
  if (!find_place<WideRow, kThreads>(a, (int)gridDim.x, scan, found, header, place)) return;
  const int id = place.id;
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
    const int wave_all = base + row_first + (in_row + wave * 32) / a.group + 1;                 // keys that all of the wave's columns see
    const int k_begin = first ? 0 : __builtin_amdgcn_readfirstlane(s.keys_at(from));
    const int k_end = __builtin_amdgcn_readfirstlane(last ? visible : min(s.keys_at(to), visible));

    bf16x8 qf[NKS];
    int limit;                                               // last key that the lane's column sees, less what the lane's half adds to a key's number
    {
      const int mine = wave * 32 + l32, row = row_first + (in_row + mine) / a.group, head = hk * a.group + (in_row + mine) % a.group;
      const bool real = mine < cols;
      const bf16* qp = q + ((size_t)(s.row0 + (real ? row : 0)) * a.Hq + (real ? head : 0)) * D + 8 * half;
      const unsigned flip = a.q_sign < 0.f ? 0x80008000u : 0u, keep = real && a.q_sign != 0.f ? 0xffffffffu : 0u;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        uint4 w = *reinterpret_cast<const uint4*>(qp + 16 * ks);
        w.x = (w.x ^ flip) & keep; w.y = (w.y ^ flip) & keep; w.z = (w.z ^ flip) & keep; w.w = (w.w ^ flip) & keep;
        qf[ks] = __builtin_bit_cast(bf16x8, w);
      }
      limit = real ? base + row - 4 * half : -64;
    }
    float m = limit == -64 ? 0.f : -INFINITY, l = 0.f;       // the reference (log2 units), the sum against it
    floatx16 oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;

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
      // second half's O^T products; a half's probabilities are formed beside the products that follow its scores.  A half is 32 keys.
      // Fragments are read kAhead ahead of their products.
      auto tile = [&](auto buf_, Stage<D>& x, const int k0) {
        constexpr int BUF = decltype(buf_)::value, NF = 2 * NKS, NV = 4 * NDB, kAhead = 4;
        const bool masked = there != 15 || k0 + kKeys > wave_all;
        auto mask = [&](floatx16& s, int kb) {               // key 32 kb + 8 (r / 4) + 4 half + r % 4 of the tile
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kb + 8 * (r >> 2) + (r & 3) > limit - k0 || !(there >> (2 * kb + (r >> 3)) & 1)) s[r] = -INFINITY;
        };
        floatx16 sacc[2];
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
        unsigned pf[2][8];
        float sum = 0.f, y = 0.f, ref = 0.f;
        auto probability = [&](auto kb_, const floatx16& s, int e) {
          constexpr int kb = decltype(kb_)::value;
          const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale_log2, -ref));
          sum = e == 0 ? z : sum + z;
          if (e & 1) {
            typedef float float2v __attribute__((ext_vector_type(2)));
            unsigned w = __builtin_bit_cast(unsigned, __builtin_convertvector((float2v){y, z}, bf16x2v));
            asm volatile("" : "+v"(w));                      // (packed here: not the two floats kept)
            pf[kb][e >> 1] = w;
          }
          y = z;
        };
        // A half's reference: it moves (rarely) where a lane's sum gets large, and from -inf at the first key that is seen; the half's scores and
        // probabilities are formed again.  (Scores kept for this case would cost registers in every tile.)
        auto settle = [&](auto kb_) {
          constexpr int kb = decltype(kb_)::value;
          if (__builtin_expect(__any(!(sum <= kLazySum) || m == -INFINITY), 0)) {
            floatx16 s;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) s = mfma32(*(LDS_PTR(const bf16x8))(pk + kb * 32 * kKRow<D> + ks * 32), qf[ks], s);
            if (masked) mask(s, kb);
            float mx = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
            mx = fmaxf(mx, xor32(mx)) * a.scale_log2;
            const float to_m = fmaxf(m, mx), alpha = to_m == m ? 1.f : __builtin_amdgcn_exp2f(m - to_m);
            m = to_m;
            l *= alpha;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
              for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
            ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int e = 0; e < 16; ++e) probability(kb_, s, e);
          }
          l += sum;
        };
        auto weights = [&](int j) {
          typedef unsigned uint4v __attribute__((ext_vector_type(4)));
          const unsigned* w = &pf[j >> 1][4 * (j & 1)];
          return __builtin_bit_cast(bf16x8, (uint4v){w[0], w[1], w[2], w[3]});
        };
        // a half's 16 probabilities beside products 2 .. NKS - 1 (the scores are still on their way beside the first two)
        auto share = [&](auto kb_, auto i_) {
          constexpr int i = decltype(i_)::value, n = NKS - 2;
          if constexpr (i >= 2)
            static_for<(i - 2) * 16 / n, (i - 1) * 16 / n>([&](auto e_) { probability(kb_, sacc[decltype(kb_)::value], decltype(e_)::value); });
        };
        const int bad = clean_scales<D>(x, k0 + kKeys, visible);
        bf16x4 part;
        static_for<0, kAhead>([&](auto o_) { issue(o_); });
        static_for<0, NKS>([&](auto i_) {
          constexpr int i = decltype(i_)::value;
          wait_frag<later(i)>(kf[i]);
          if constexpr (i < NKS / 2) unpack_slot<D>(x, uk, uv, i, part);
          if constexpr (i == 0) {
            const floatx16 zero = {};
            sacc[0] = mfma32(kf[i], qf[i], zero);
          } else {
            sacc[0] = mfma32(kf[i], qf[i], sacc[0]);
          }
          issue(IC<i + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        if (masked) mask(sacc[0], 0);
        ref = m == -INFINITY ? 0.f : m;
        static_for<0, NKS>([&](auto i_) {
          constexpr int i = decltype(i_)::value, o = NKS + i;
          wait_frag<later(o)>(kf[o]);
          share(IC<0>{}, i_);
          if constexpr (i == 0) {
            const floatx16 zero = {};
            sacc[1] = mfma32(kf[o], qf[i], zero);
          } else {
            sacc[1] = mfma32(kf[o], qf[i], sacc[1]);
          }
          issue(IC<o + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        settle(IC<0>{});
        if (masked) mask(sacc[1], 1);
        static_for<0, 2 * NDB>([&](auto i_) {
          constexpr int i = decltype(i_)::value;
          wait_frag<later(NF + i)>(vf[i][0], vf[i][1]);
          share(IC<1>{}, i_);
          oacc[i % NDB] = mfma32(join_frag(vf[i][0], vf[i][1]), weights(i / NDB), oacc[i % NDB]);
          issue(IC<NF + i + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        settle(IC<1>{});
        LDS_PTR(const int) info = (LDS_PTR(const int))(lds + kBadAt<D> + BUF * kBadBytes);
        int any_bad = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) any_bad |= info[w];
        static_for<0, 2 * NDB>([&](auto i_) {
          constexpr int i = decltype(i_)::value, p = 2 * NDB + i;
          wait_frag<later(NF + p)>(vf[p][0], vf[p][1]);
          if constexpr (i < NKS / 2) unpack_slot<D>(x, uk, uv, NKS / 2 + i, part);
          oacc[i % NDB] = mfma32(join_frag(vf[p][0], vf[p][1]), weights(2 + i / NDB), oacc[i % NDB]);
          issue(IC<NF + p + kAhead>{});
          __builtin_amdgcn_sched_barrier(0);
        });
        note_bad<D>(lds, BUF ^ 1, bad);
        if (__builtin_amdgcn_readfirstlane(any_bad)) {       // scales that are not finite: NaN where their keys are seen
          int hit = 0;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int key = 32 * kb + 8 * (r >> 2) + (r & 3);
              hit |= info[(key + 4 * half) >> 3] && k0 + key <= limit ? info[kWaves + key + 4 * half] : 0;
            }
          hit |= __shfl_xor(hit, 32);
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const float poison = hit & (256 | 1 << db) ? __builtin_nanf("") : 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[db][r] += poison;
          }
          l += hit & 256 ? __builtin_nanf("") : 0.f;
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
    // (the column again, from a copy of the thread's number: its places in the outputs would otherwise be kept in registers through the walk)
    const int me = thread_number(), out_half = me >> 5 & 1, col = (me >> 6) * 32 + (me & 31);
    const int out_row = row_first + (in_row + col) / a.group, out_head = hk * a.group + (in_row + col) % a.group;
    l += xor32(l);
    if (col < cols && first && last) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* op = o + ((size_t)(s.row0 + out_row) * a.Hq + out_head) * D + 4 * out_half;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : oacc[db][r + e] * inv;
          store_out<4>(op + 32 * db + 2 * r, x);
        }
      if (lse && out_half == 0) lse[(size_t)out_head * a.c.n_rows + s.row0 + out_row] = (m + __builtin_amdgcn_logf(l)) * kLn2;
    } else if (!(first && last)) {
      float* part = part_of<D>(ws + parts_at, id, first ? 1 : 0);
      if ((me >> 6) * 32 < cols) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<floatx4v*>(part + part_at<D>(me >> 6, db, r >> 2, me & 63)) = floatx4v{oacc[db][r], oacc[db][r + 1], oacc[db][r + 2], oacc[db][r + 3]};
        if (out_half == 0) { part[kCols * D + col] = m; part[kCols * D + kCols + col] = l; }
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

// Adds up the parts of the split item listed at blockIdx.x, in order.  A wave has the 64 lanes of eight channels of a wave's columns, as they were
// stored: blockIdx.y = wave of the item's block, then 32 channels; then 8 channels, by the waves of a block (RUNS = 1) or by blockIdx.z (RUNS = 4: each
// wave adds up a run of the parts).  128 parts of two items: 13 us with four runs, 22 with one; 8 parts of 32 items: 12.5 and 10.
template <int D, int RUNS>
__global__ __launch_bounds__(256) void cache_attn_wide_join_kernel(AttnArgs a, bf16* __restrict__ o, float* __restrict__ lse, char* __restrict__ ws, size_t parts_at) {
  Header* header = split_header(ws + kListBytes);
  const Split s = split_list(header)[blockIdx.x];            // (with the count, not behind it: the list has room for every block)
  const int wave = blockIdx.y / (D / 32), db = blockIdx.y % (D / 32), r4 = RUNS == 1 ? threadIdx.x >> 6 : blockIdx.z, run = RUNS == 1 ? 0 : threadIdx.x >> 6;
  const int lane = threadIdx.x & 63, c = wave * 32 + (lane & 31);
  if ((int)blockIdx.x >= header->listed || s.parts == 0 || wave * 32 >= s.cols) return;
  const int each = (s.parts + RUNS - 1) / RUNS, begin = min(run * each, s.parts), end = min(begin + each, s.parts);
  auto part = [&](int p) { return part_of<D>(ws + parts_at, s.first + p, p == 0 ? 1 : 0); };
  float m = -INFINITY;
#pragma unroll 8
  for (int p = begin; p < end; ++p) m = fmaxf(m, part(p)[kCols * D + c]);
  float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  floatx4v x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = begin; p < end; ++p) {
    const float* y = part(p);
    const float f = __builtin_amdgcn_exp2f(y[kCols * D + c] - ref);
    l = __builtin_fmaf(y[kCols * D + kCols + c], f, l);
    x += *reinterpret_cast<const floatx4v*>(y + part_at<D>(wave, db, r4, lane)) * f;
  }
  if constexpr (RUNS > 1) {
    __shared__ float ms[RUNS][64], ls[RUNS][64];
    __shared__ floatx4v xs[RUNS][64];
    ms[run][lane] = m, ls[run][lane] = l, xs[run][lane] = x;
    __syncthreads();
    if (run != 0) return;
#pragma unroll
    for (int i = 1; i < RUNS; ++i) m = fmaxf(m, ms[i][lane]);
    ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
    x = floatx4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const float f = __builtin_amdgcn_exp2f(ms[i][lane] - ref);
      l = __builtin_fmaf(ls[i][lane], f, l);
      x += xs[i][lane] * f;
    }
  }
  if (c >= s.cols) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int r = s.row0 + (s.col0 + c) / a.group, hd = s.head0 + (s.col0 + c) % a.group, e = 32 * db + 8 * r4 + 4 * (lane >> 5);
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
    if (a.slots && 16 * a.slots <= blocks)   // 16 parts of an item or more
      hipLaunchKernelGGL((cache_attn_wide_join_kernel<D, 4>), dim3(a.slots, kWaves * (D / 32), 4), dim3(256), 0, (hipStream_t)stream, a, (bf16*)o, lse,
                         (char*)ws, parts_at);
    else
      hipLaunchKernelGGL((cache_attn_wide_join_kernel<D, 1>), dim3(a.slots ? a.slots : blocks, kWaves * (D / 32)), dim3(256), 0, (hipStream_t)stream, a, (bf16*)o, lse,
                         (char*)ws, parts_at);
    return (int)hipGetLastError();
  };
  return p.head_dim == 128 ? run(IC<128>{}) : run(IC<64>{});
}

}  // namespace slimattn
