// Rotary positions, and new keys and values into a paged cache (keys turned on the way), on gfx950.
//
// Pair (x0, x1) of a head turns by the angle a = position * frequency:  y0 = A (x0 cos a - x1 sin a),  y1 = A (x0 sin a + x1 cos a).
// Bound by memory: every element is read once and written once, 6 operations a pair.  A thread owns one piece of a token's head (16
// bytes of it where rows allow; with the half layout the two pieces that hold the partners) and forms its sines and cosines ONCE for all
// heads of the token that its workgroup handles, four heads' loads in flight.  The angle is reduced in 64 bits, in full turns: a
// position times a frequency in 32 bits is off by 2^-24 of the angle, 0.06 radians at a million; the multiplication, the nearest whole turn
// and the difference are three fp64 instructions a pair, and what is left is at most half a turn, for which 32 bits are enough.  (The frequency in turns
// and the product are rounded once each: 2^-52 of the angle, as much as fp32's rounding from 2^28 radians on.)
// q and k of 32,760 tokens, 12 heads of 128 each, bf16 (403 MB): 81 us, 5.0 TB/s, the rate of a large copy; two frames of 3 streams into pages (93 MB)
// 18.4 us (21 with the host's share of a call); 24 tokens 6.8 us (9), a chain of dependent loads.
#include "seq.h"

namespace vm {

namespace {

constexpr int THREADS = 256;

template <typename E, int V>
struct alignas(sizeof(E) * V) Piece {
  E e[V];
};

template <typename E, int V, bool HALF, bool APPEND>
__global__ void __launch_bounds__(THREADS) rotary_kernel(RotaryParams P, RotaryTurns F, int units, int tokens_per_block, int heads_per_block) {
  // units of a token's head: with turned pairs first the pieces that hold them, then the pieces that pass through
  const int which = APPEND ? (int)(blockIdx.y & 1) : 0;
  const int first_head = (APPEND ? blockIdx.y >> 1 : blockIdx.y) * heads_per_block;
  const int t_local = threadIdx.x / units;
  const int unit = threadIdx.x - t_local * units;
  const long long token = (long long)blockIdx.x * tokens_per_block + t_local;
  int lo = 0, begin = 0, end = 0;  // append: the token's sequence, the last that begins at or before it
  if (APPEND) {
    const int n = P.n_seqs;
    const int tok = (int)min(token, (long long)P.tokens - 1);
    if (n < 64) {  // the wave holds all starts
      const int lane = threadIdx.x & 63;
      const int mine = P.starts[min(lane, n)];
#pragma unroll
      for (int step = 32; step > 0; step /= 2) {
        const int at = __shfl(mine, min(lo + step, 63));
        if (lo + step < n && at <= tok) lo += step;
      }
      begin = __shfl(mine, lo);
      end = __shfl(mine, lo + 1);
    } else {
      int hi = n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (P.starts[mid] <= tok) lo = mid;
        else hi = mid;
      }
      begin = P.starts[lo];
      end = P.starts[lo + 1];
    }
    end = min(end, P.tokens);
  }
  if (t_local >= tokens_per_block || token >= P.tokens) return;

  long long slot_off[2] = {0, 0};  // append: where the token's slot lies in the caches of keys and of values
  int at = 0;
  if (APPEND) {
    if (token < begin || token >= end) return;
    const long long room = (long long)P.table_width * P.page_size;
    const long long have = min((long long)max(P.lengths[lo], 0), room);
    const long long p = have - ((long long)end - token);
    if (p < 0) return;
    at = (int)p;
    const int page = P.table[lo * P.table_stride + at / P.page_size];
    if (page < 0 || page >= P.n_pages) return;
    const int slot = at % P.page_size;
#pragma unroll
    for (int x = 0; x < 2; ++x) slot_off[x] = page * P.out_page[x] + slot * P.out_t[x];
  }

  const int pairs = P.turned[which];
  // units with turned pairs (V = 1, interleaved: a unit is a pair; wide: the last may hold pairs that are not turned)
  const int turning_units = HALF ? pairs / V : V == 1 ? pairs : (2 * pairs + V - 1) / V;
  const bool turns = unit < turning_units;
  int c0, c1 = 0;  // channels of the unit's pieces
  constexpr int NP = V == 1 ? 1 : HALF ? V : V / 2;  // pairs of a unit
  float cs[NP], sn[NP];
  if (turns) {
    c0 = HALF ? unit * V : V == 1 ? 2 * unit : unit * V;
    c1 = HALF ? c0 + pairs : c0 + 1;
    const int first = HALF ? unit * V : V == 1 ? unit : unit * (V / 2);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int pair = min(first + i, pairs - 1);
      const int axis = (pair >= P.axis_end[0]) + (pair >= P.axis_end[1]);
      const int pos = P.positions ? P.positions[axis * P.axis_stride + token] : at;
      const double turn = (double)pos * F.per_position[pair];
      const float rest = (float)(turn - __builtin_rint(turn));
      float s, c;
      sincospif(2.0f * rest, &s, &c);
      cs[i] = P.amplitude * c;
      sn[i] = P.amplitude * P.sign * s;
    }
  } else {
    c0 = (HALF || V == 1 ? 2 * pairs : turning_units * V) + (unit - turning_units) * V;
    if (c0 >= P.d) return;  // (keys and values of one launch need not have as many units)
  }

  const int all = P.heads[0] + (APPEND ? 0 : P.heads[1]);
  const int last = min(first_head + heads_per_block, all);
  auto source = [&](int h) -> const E* {
    const int x = APPEND ? which : h >= P.heads[0];
    const int hh = !APPEND && x ? h - P.heads[0] : h;
    return (const E*)P.in[x] + token * P.in_t[x] + hh * P.in_h[x];
  };
  auto target = [&](int h) -> E* {
    const int x = APPEND ? which : h >= P.heads[0];
    const int hh = !APPEND && x ? h - P.heads[0] : h;
    return (E*)P.out[x] + (APPEND ? slot_off[x] : token * P.out_t[x]) + hh * P.out_h[x];
  };
  constexpr int U = 4;
  constexpr bool TWO = HALF || V == 1;  // a unit is two pieces
  for (int h0 = first_head; h0 < last; h0 += U) {
    Piece<E, V> a[U], b[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const E* s = source(min(h0 + i, last - 1));
      a[i] = *reinterpret_cast<const Piece<E, V>*>(s + c0);
      if (TWO && turns) b[i] = *reinterpret_cast<const Piece<E, V>*>(s + c1);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (h0 + i >= last) break;
      E* o = target(h0 + i);
      if (turns) {
        if (TWO) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float x0 = load_f<E>(&a[i].e[e]), x1 = load_f<E>(&b[i].e[e]);
            const int j = V == 1 ? 0 : e;
            store_f<E>(&a[i].e[e], x0 * cs[j] - x1 * sn[j]);
            store_f<E>(&b[i].e[e], x0 * sn[j] + x1 * cs[j]);
          }
          *reinterpret_cast<Piece<E, V>*>(o + c1) = b[i];
        } else {
#pragma unroll
          for (int j = 0; j < V / 2; ++j) {
            if (c0 / 2 + j >= pairs) break;  // the rest of a piece passes through
            const float x0 = load_f<E>(&a[i].e[2 * j]), x1 = load_f<E>(&a[i].e[(2 * j + 1) % V]);
            store_f<E>(&a[i].e[2 * j], x0 * cs[j] - x1 * sn[j]);
            store_f<E>(&a[i].e[(2 * j + 1) % V], x0 * sn[j] + x1 * cs[j]);
          }
        }
      }
      *reinterpret_cast<Piece<E, V>*>(o + c0) = a[i];
    }
  }
}

template <typename E, int V>
hipError_t launch(const RotaryParams& P, const RotaryTurns& F, hipStream_t st) {
  const bool append = P.starts != nullptr;
  const bool half = !P.interleaved;
  int units = 0;
  for (int x = 0; x < (append ? 2 : 1); ++x) {
    const int n = P.turned[x];
    const int turning = half ? n / V : V == 1 ? n : (2 * n + V - 1) / V;
    const int u = turning + (P.d - (half || V == 1 ? 2 * n : turning * V)) / V;
    if (u > units) units = u;
  }
  const int tokens_per_block = THREADS / units;
  const long long blocks = ((long long)P.tokens + tokens_per_block - 1) / tokens_per_block;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  const int heads = append ? P.heads[0] : P.heads[0] + P.heads[1];
  // All heads of a token in one workgroup spare sines; a launch short of four workgroups on every compute unit spreads its heads.
  int split = 1;
  while (split * 4 < heads && blocks * split < 4LL * compute_units()) split *= 2;
  const int per = (heads + split - 1) / split;
  const dim3 grid((unsigned)blocks, (unsigned)((heads + per - 1) / per * (append ? 2 : 1)));
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(THREADS), 0, st, P, F, units, tokens_per_block, per);
    return hipGetLastError();
  };
  if (append) return half ? go(rotary_kernel<E, V, true, true>) : go(rotary_kernel<E, V, false, true>);
  return half ? go(rotary_kernel<E, V, true, false>) : go(rotary_kernel<E, V, false, false>);
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& P, const RotaryTurns& F, int elem_bytes, bool wide, hipStream_t st) {
  if (elem_bytes == 2) return wide ? launch<bf16_t, 8>(P, F, st) : launch<bf16_t, 1>(P, F, st);
  return wide ? launch<float, 4>(P, F, st) : launch<float, 1>(P, F, st);
}

}  // namespace vm
