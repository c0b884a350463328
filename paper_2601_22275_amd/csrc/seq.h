// Declarations shared by the token-sequence units (rotary.hip, seq_*.hip; not part of the ABI).
#pragma once
#include "../../include/vmonarch_sequence.h"
#include <atomic>

#include "common.h"

namespace vm {

// api.hip: the library's error text and workspaces
int api_fail(int code, const char* fmt, ...);
void* api_workspace(size_t bytes, int* err, void* call_ws, size_t call_ws_bytes, hipStream_t st);

// A strided token tensor on the device
template <typename E>
struct Rows {
  E* p;
  long long t, h;  // elements between tokens, between heads
};

// Keys or values: packed (page_size 0), or in pages
template <typename E>
struct KeyRows {
  const E* p;
  long long t, h, page;
};

// One attention problem as the kernels see it.  Query rows are PACKED: row r of a sequence and key head is token r / group of it, query
// head kv_head * group + r % group, so that the heads that share keys fill a tile together, single tokens as well as prompts.
template <typename E>
struct SeqParams {
  Rows<const E> q;
  KeyRows<E> k, v;
  Rows<E> out;
  float* lse;           // [heads_q][tokens_q], or null
  const int* q_starts;
  const int* k_starts;  // packed keys
  const int* lengths;   // keys in pages
  const int* table;
  long long table_stride;
  int table_width, page_size, n_pages;  // page_size 0: packed keys
  int n_seqs;
  int tokens_q, tokens_k;
  int heads_kv, group, d;
  int causal;
  int aligned;          // rows on 16-byte boundaries, d a multiple of 16 bytes
  float scale;
  // backward
  Rows<const E> o, d_out;
  Rows<E> dq, dk, dv;
  float* delta;         // per row: seq_general.hip d_out . out, [heads_q][tokens_q]; seq_bwd.hip see there
  // ranges of keys (forward, pages) or of query rows (backward): partial results and their log-sums
  float* part_o;
  float* part_s;
  int ranges;
};

// ---- device: sequences --------------------------------------------------------------------------------------------------------
struct Span {
  int seq, tile;     // tile of `BM` packed rows (keys: group 1) within the sequence
  int begin, count;  // the sequence's tokens
};

// Start of sequence s, kept inside the tensor and in order whatever the array holds
__device__ __forceinline__ int start_of(const int* starts, int s, int tokens) { return min(max(starts[s], 0), tokens); }

// Tiles of BM rows (tokens * rows_per_token) of all sequences in one row of workgroups.  Sequence s owns tiles f(s) .. f(s+1) - 1 with
// f(s) = floor(starts[s] rows_per_token / BM) + s: at least the ceil(rows / BM) it needs, and the last one needs none from
// ceil(tokens rows_per_token / BM) + n - 1 on: the host launches that many without seeing the lengths.  The sequence of tile `t` is found by all
// lanes of a wave at once.
__device__ __forceinline__ Span find_tile(const int* starts, int n_seqs, int tokens, int rows_per_token, int BM, int t) {
  const int lane = threadIdx.x & 63;
  int s = 0;
  for (int base = 0; base < n_seqs; base += 64) {
    const int i = base + lane;
    const bool at_or_before = i < n_seqs && (long long)start_of(starts, i, tokens) * rows_per_token / BM + i <= t;
    const unsigned long long b = __ballot(at_or_before);
    if (b == 0) break;
    s = base + 63 - __builtin_clzll(b);
    if (s != base + 63) break;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  Span w;
  w.seq = s;
  w.begin = start_of(starts, s, tokens);
  w.count = max(start_of(starts, s + 1, tokens) - w.begin, 0);
  w.tile = t - (int)((long long)w.begin * rows_per_token / BM + s);
  if (w.tile < 0) w.tile = w.count = 0;  // tokens in front of the first sequence
  return w;
}

// The same tiles in order of their work under a causal mask, most first, for up to 64 sequences: with n_s tiles in sequence s, tile r - 1 sees (as
// queries; as keys, tile n_s - r is seen by) r tiles' worth, so the order is by r, all sequences together.  Above r lie G(r) = sum_s max(n_s - r, 0)
// tiles.  Sequences one after another leave the card waiting for the last long one (3 x 4096 tokens, 12 heads on 4, d = 128, forward and backward:
// 730 -> 692 us; 7 prompts of up to 5000 346 -> 304).  `tile` is r - 1 here.
__device__ __forceinline__ Span find_tile_by_work(const int* starts, int n_seqs, int tokens, int rows_per_token, int BM, int t) {
  const int lane = threadIdx.x & 63;
  int begin = 0, count = 0;
  if (lane < n_seqs) {
    begin = start_of(starts, lane, tokens);
    count = max(start_of(starts, lane + 1, tokens) - begin, 0);
  }
  const int n = (int)(((long long)count * rows_per_token + BM - 1) / BM);
  auto above = [&](int r) {
    int x = max(n - r, 0);
#pragma unroll
    for (int step = 1; step < 64; step *= 2) x += __shfl_xor(x, step);
    return __builtin_amdgcn_readfirstlane(x);
  };
  Span w = {0, 0, 0, 0};
  int most = n;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) most = max(most, __shfl_xor(most, step));
  most = __builtin_amdgcn_readfirstlane(most);
  if (t >= above(0)) return w;
  int lo = 0, hi = most;  // G(lo) > t >= G(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (above(mid) > t) lo = mid;
    else hi = mid;
  }
  const int nth = t - above(hi);
  const unsigned long long have = __ballot(n >= hi);
  // the sequence with `nth` others of as many tiles in front of it
  const bool here = n >= hi && __builtin_popcountll(have & ((1ull << lane) - 1)) == nth;
  w.seq = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(__ballot(here)));
  w.begin = __shfl(begin, w.seq);
  w.count = __shfl(count, w.seq);
  w.begin = __builtin_amdgcn_readfirstlane(w.begin);
  w.count = __builtin_amdgcn_readfirstlane(w.count);
  w.tile = hi - 1;
  return w;
}

// Upper bound of the tiles of all sequences (see find_tile); one sequence: what it needs
inline long long tile_bound(long long tokens, int rows_per_token, int BM, int n_seqs) { return (tokens * rows_per_token + BM - 1) / BM + n_seqs - 1; }

// Keys of sequence s: where they begin (packed) and how many there are
template <typename E>
__device__ __forceinline__ int keys_of(const SeqParams<E>& P, int s, int* begin) {
  if (P.page_size > 0) {
    *begin = 0;
    const long long room = (long long)P.table_width * P.page_size;
    return (int)min((long long)max(P.lengths[s], 0), room);
  }
  *begin = start_of(P.k_starts, s, P.tokens_k);
  return max(start_of(P.k_starts, s + 1, P.tokens_k) - *begin, 0);
}

// Lets a kernel use `bytes` of LDS on the current device; done: which devices have it already
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<unsigned long long>* done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev < 64 && (done->load(std::memory_order_acquire) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done->fetch_or(bit, std::memory_order_release);
  return e;
}

// ---- launchers (host) -----------------------------------------------------------------------------------------------------------
struct RotaryParams {
  const void* in[2];   // q, k (append: k, v)
  void* out[2];
  long long in_t[2], in_h[2], out_t[2], out_h[2], out_page[2];
  int heads[2];
  int turned[2];       // pairs turned in tensor 0 / 1 (append: values pass through)
  int tokens, d;
  const int* positions;  // [axes][tokens]; null: the position in the sequence (append)
  long long axis_stride;
  int axis_end[3];     // pairs below this one belong to the axis
  int interleaved;
  float amplitude;
  float sign;          // of the sine
  // append
  const int* starts;
  const int* lengths;
  const int* table;
  long long table_stride;
  int table_width, page_size, n_pages, n_seqs;
};
struct RotaryTurns {
  double per_position[VMONARCH_ROTARY_MAX_PAIRS];  // full turns: frequency / 2 pi
};
// rotary.hip; elem_bytes 2: bf16, 4: float32; wide: rows in 16-byte pieces
hipError_t launch_rotary(const RotaryParams& P, const RotaryTurns& F, int elem_bytes, bool wide, hipStream_t st);

// seq_mfma.hip : bf16, aligned rows, d <= D (compiled for D = 64 and 128)
template <int D>
hipError_t launch_seq_attention_mfma(const SeqParams<bf16_t>& P, hipStream_t st);
// seq_token.hip : the same for few rows (pages), and the join of ranges for everything that is cut into them
template <int D>
hipError_t launch_seq_token(const SeqParams<bf16_t>& P, hipStream_t st);
template <typename E>
hipError_t launch_seq_join(const SeqParams<E>& P, hipStream_t st);
// Channels of a partial result's row
inline int seq_padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// seq_bwd.hip : the backward pass, bf16, aligned rows, d <= D (ranges: of query rows, for dK and dV; part_o their partial sums)
int seq_bwd_ranges(int n_seqs, long long tokens_q, long long tokens_k, int heads_kv, int group);
template <int D>
hipError_t launch_seq_bwd_mfma(const SeqParams<bf16_t>& P, hipStream_t st);

// seq_general.hip : any d <= 256, any strides, on the fp32 matrix units
template <typename E>
hipError_t launch_seq_attention_general(const SeqParams<E>& P, hipStream_t st);
template <typename E>
hipError_t launch_seq_attention_bwd_general(const SeqParams<E>& P, hipStream_t st);

}  // namespace vm
