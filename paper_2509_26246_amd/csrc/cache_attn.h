// Attention over the 4-bit cache: what its kernels share -- the row of work that a launch divides evenly among its blocks, whatever the lengths
// are, and the list of items whose parts have to be added up afterwards.
#pragma once
#include "block_order.h"
#include "cache.h"

namespace slimattn {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxGrid = 1024;       // at most four blocks per compute unit

typedef float floatx4v __attribute__((ext_vector_type(4)));

struct AttnArgs {
  CacheView c;
  int group, Hq;                     // query heads per KV head; of all
  float scale_log2;                  // > 0
  float q_sign;                      // scale < 0 turns q around; 0 makes it zero
  long long narrow_cols;             // sequences of more query columns (rows x group) than this are the wide kernel's
  int slots;                         // split items are listed by number if there are at most this many items, 0: by the block that began them
};

// An item that blocks share, written by the one that holds its start for the launch that adds its parts up (parts = 0: not shared).
struct Split { int first, parts, row0, cols, col0, head0, pad[2]; };
struct Header { int listed, pad[7]; };   // entries that were written
constexpr size_t kListBytes = sizeof(Header) + kMaxGrid * sizeof(Split);   // of each kernel, narrow first, at the workspace's start
__device__ __forceinline__ Header* split_header(char* ws) { return reinterpret_cast<Header*>(ws); }
__device__ __forceinline__ Split* split_list(Header* h) { return reinterpret_cast<Split*>(h + 1); }

__device__ __forceinline__ unsigned word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ unsigned word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }
__device__ __forceinline__ unsigned word(unsigned v, int) { return v; }

// Rows of a sequence among the tensors' rows, and its length.
__device__ __forceinline__ void seq_rows(const AttnArgs& a, int b, int& row0, int& rows, int& len) {
  row0 = b;
  rows = 1;
  if (a.c.row_ptr) {
    row0 = min(max(a.c.row_ptr[b], 0), a.c.n_rows);
    rows = min(max(a.c.row_ptr[b + 1], row0), a.c.n_rows) - row0;
  }
  len = seq_len(a.c, b);
}

__device__ __forceinline__ long long wave_scan(long long x) {   // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = __shfl_up(x, d);
    if ((int)(threadIdx.x & 63) >= d) x += y;
  }
  return x;
}

// Inclusive scan over the block of THREADS; `total` gets the sum.
template <int THREADS>
__device__ __forceinline__ long long block_scan(long long x, long long* lds, long long& total) {
  x = wave_scan(x);
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[wave] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) x += lds[w];
    total += lds[w];
  }
  return x;
}

// The block that holds unit x of U, when block i of n holds units [U i / n, U (i + 1) / n).
__device__ __forceinline__ int block_of(long long x, long long U, int n) { return (int)(((x + 1) * n - 1) / U); }

// Piece `id` of the work: units [begin, end) of `total`, divided among `blocks` blocks; the sequence in which it begins, with the units and
// items before that sequence.
struct Place {
  long long total, begin, end, seq_begin, seq_item;
  int blocks, id, seq;
};

// Row: what a sequence adds (units_of_all(), items()), and how many blocks share a row of so much work.  False: nothing to do for this block.
// As many sequences as the block has threads are one look at the lengths.  N: the launch's blocks.
template <class Row, int THREADS>
__device__ __forceinline__ bool find_place(const AttnArgs& a, int N, long long* scan, long long* found, Header* header, Place& p) {
  const int tid = threadIdx.x;
  const bool one_look = a.c.n_seqs <= THREADS, with_items = Row::kNeedsItems || a.slots;
  long long mine = 0, my_items = 0, items = 0;
  for (int b = tid; b < a.c.n_seqs; b += THREADS) {
    const Row s(a, b);
    mine += s.units_of_all();
    my_items += s.items();
  }
  const long long units_to = block_scan<THREADS>(mine, scan, p.total), items_to = with_items ? block_scan<THREADS>(my_items, scan, items) : 0;
  p.blocks = Row::blocks(a, N, p.total, items);
  if (blockIdx.x == 0 && tid == 0) header->listed = a.slots ? (int)min((long long)a.slots, items) : p.blocks;
  if ((int)blockIdx.x >= p.blocks) return false;
  p.id = piece_of_block(blockIdx.x, p.blocks);
  p.begin = p.total * p.id / p.blocks;
  p.end = p.total * (p.id + 1) / p.blocks;
  if (one_look) {
    if (p.begin < units_to && p.begin >= units_to - mine) { found[0] = tid; found[1] = units_to - mine; found[2] = items_to - my_items; }
  } else {
    long long units_before = 0, items_before = 0;
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += THREADS) {       // (begin < total: some sequence has it)
      const int b = b0 + tid;
      long long w = 0, i = 0, units = 0, n = 0;
      if (b < a.c.n_seqs) {
        const Row s(a, b);
        w = s.units_of_all();
        i = s.items();
      }
      const long long end = units_before + block_scan<THREADS>(w, scan, units), item_end = with_items ? items_before + block_scan<THREADS>(i, scan, n) : 0;
      if (p.begin < end && p.begin >= end - w) { found[0] = b; found[1] = end - w; found[2] = item_end - i; }
      if (p.begin < units_before + units) break;
      units_before += units;
      items_before += n;
    }
  }
  __syncthreads();
  p.seq = __builtin_amdgcn_readfirstlane((int)found[0]);
  p.seq_begin = found[1];
  p.seq_item = found[2];
  return true;
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

}  // namespace slimattn
