// Attention over packed sequences and over pages, forward and backward, on the fp32 matrix units of gfx950: any d <= 256, any strides,
// float32 or bf16 in memory.  What the bf16 kernels (seq_mfma.hip, seq_bwd.hip) do not take runs here, float32 among it.
//
// A workgroup is four waves of 16 owner rows, or twice four that take every other tile of the stream and add up at the end (one chain of work
// half as long); the other tensor's rows stream through LDS in tiles of 32, in fp32.  All products are
// v_mfma_f32_16x16x4_f32, in the form X^T = (stream rows) (owner rows)^T, so that lane (i = lane % 16, g = lane / 16) holds owner row i
// and stream rows 4 g .. + 3 of a block of 16: a softmax row's sums are per-lane scalars plus one exchange among four lanes, and
// the weights are the B operand of the next product as they stand (its k index runs over rows 4 g + r for fixed r).  The order of the
// channels within a product is free as well: a lane reads four adjacent channels at a time (16 j + 4 g .. + 3), and of a transposed
// operand the channels 64 c + 4 i .. + 3, so that every LDS read is 16 bytes wide.
// The backward pass is two launches of one kernel, as the bf16 one: rows of queries own dq, rows of keys own dk and dv; the row sums
// d_out . out come with the first and serve the second.
// Bound by the matrix units (157 TFLOP/s in fp32; a large library product reaches 154) where rows are many, by the longest chain of tiles, 2 us each
// at d = 128, where they are few.  4 ragged causal prompts of up to 1001 tokens, 10 heads on 2, d = 64, float32: 59 us (52 TFLOP/s); 9000 tokens 1181
// (88; 1418 with the owner rows waited for in the loop and a branch per key group).
#include <type_traits>

#include "seq.h"

namespace vm {

namespace {

constexpr int BM = 64;   // owner rows of a workgroup
constexpr int BN = 32;   // stream rows of a tile
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ f32x4 mfma(float a, float b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Channels c .. c + 3 of a row in fp32, zeros past d
template <typename E>
__device__ __forceinline__ f32x4 load4(const E* row, int c, int d, bool aligned) {
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (aligned) {
    if (c < d) {
      if constexpr (sizeof(E) == 4) {
        x = *reinterpret_cast<const f32x4*>(row + c);
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(row + c);
        x[0] = __uint_as_float(w.x << 16);
        x[1] = __uint_as_float(w.x & 0xffff0000u);
        x[2] = __uint_as_float(w.y << 16);
        x[3] = __uint_as_float(w.y & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < d) x[e] = load_f<E>(row + c + e);
  }
  return x;
}
template <typename E>
__device__ __forceinline__ void store4(E* row, int c, int d, bool aligned, float f0, float f1, float f2, float f3) {
  if (aligned && sizeof(E) == 4) {
    if (c < d) *reinterpret_cast<f32x4*>(row + c) = f32x4{f0, f1, f2, f3};
    return;
  }
  if (c < d) store_f<E>(row + c, f0);
  if (c + 1 < d) store_f<E>(row + c + 1, f1);
  if (c + 2 < d) store_f<E>(row + c + 2, f2);
  if (c + 3 < d) store_f<E>(row + c + 3, f3);
}

// Maximum over the four lanes of an owner row (lane % 16 alike), without a trip through LDS
__device__ __forceinline__ float across_max(float x) {
  unsigned u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  u = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

template <typename E>
__device__ __forceinline__ const E* key_row(const SeqParams<E>& P, const KeyRows<E>& K, int seq, int begin, int kvh, int j) {
  if (P.page_size == 0) return K.p + (long long)(begin + j) * K.t + kvh * K.h;
  const int n = j / P.page_size;
  int page = P.table[seq * P.table_stride + n];
  if (page < 0 || page >= P.n_pages) page = 0;
  return K.p + page * K.page + (long long)(j - n * P.page_size) * K.t + kvh * K.h;
}

enum { FORWARD = 0, GRAD_Q = 1, GRAD_KV = 2 };

// Halves of a workgroup (a wave of d = 256 needs more registers than eight waves have each)
template <int D>
constexpr int parts() {
  return D == 256 ? 1 : 2;
}

template <typename E, int D, int MODE>
__global__ void __launch_bounds__(256 * parts<D>(), D == 256 ? 1 : 2) seq_general_kernel(SeqParams<E> P) {
  constexpr int LS = D + 4;          // floats of an LDS row: 16 rows of four channels fall on all banks
  constexpr int NJ = D / 16;         // 16-channel groups of a contraction over channels
  constexpr int NC = D / 64;         // 64-channel groups of an output row
  constexpr bool BWD = MODE != FORWARD;
  // d_out . out from stored rows of bf16 carries their rounding, which the difference dP - D does not forgive where a row's weight sits on a few keys
  // (on one: dP - D is zero): D = sum_j P dP in a round of its own.
  constexpr bool SUM_D = MODE == GRAD_Q && sizeof(E) == 2;
  constexpr int PARTS = parts<D>();
  __shared__ __attribute__((aligned(16))) float tiles_lds[PARTS][2][BN][LS];
  __shared__ float st_lds[PARTS][2][MODE == GRAD_KV ? BN : 1];
  const int part = threadIdx.x / 256, tid = threadIdx.x % 256;
  float (&x1)[BN][LS] = tiles_lds[part][0];  // keys (GRAD_KV: queries)
  float (&x2)[BN][LS] = tiles_lds[part][1];  // values (GRAD_KV: d_out)
  float (&st_lse)[MODE == GRAD_KV ? BN : 1] = st_lds[part][0], (&st_delta)[MODE == GRAD_KV ? BN : 1] = st_lds[part][1];
  const int lane = tid & 63, wave = tid >> 6, li = lane & 15, g = lane >> 4;
  const int kvh = blockIdx.y;
  const int group = P.group, d = P.d;
  const bool al = P.aligned;

  const int* own_starts = MODE == GRAD_KV ? P.k_starts : P.q_starts;
  const int own_tokens = MODE == GRAD_KV ? P.tokens_k : P.tokens_q, per_token = MODE == GRAD_KV ? 1 : group;
  const bool by_work = P.causal && P.n_seqs <= 64;
  Span w = by_work ? find_tile_by_work(own_starts, P.n_seqs, own_tokens, per_token, BM, blockIdx.x)
                   : find_tile(own_starts, P.n_seqs, own_tokens, per_token, BM, gridDim.x - 1 - blockIdx.x);
  if (MODE == GRAD_KV && by_work) w.tile = max((w.count + BM - 1) / BM - 1 - w.tile, 0);
  int q_begin, nq, k_begin, nk;
  if (MODE == GRAD_KV) {
    k_begin = w.begin;
    nk = w.count;
    q_begin = start_of(P.q_starts, w.seq, P.tokens_q);
    nq = max(start_of(P.q_starts, w.seq + 1, P.tokens_q) - q_begin, 0);
  } else {
    q_begin = w.begin;
    nq = w.count;
    nk = keys_of(P, w.seq, &k_begin);
  }
  const long long rows = (long long)nq * group;  // packed query rows
  const long long owners = MODE == GRAD_KV ? nk : rows;
  const long long o0 = (long long)w.tile * BM;
  if (o0 >= owners) return;
  const int more = nk - nq;  // query token i sees keys below more + 1 + i
  auto q_row = [&](const Rows<const E>& X, long long r) -> const E* {
    const int tok = (int)(r / group);
    return X.p + (long long)(q_begin + tok) * X.t + (kvh * group + (int)(r - (long long)tok * group)) * X.h;
  };
  auto stat_of = [&](long long r) -> long long {
    const int tok = (int)(r / group);
    return (long long)(kvh * group + (int)(r - (long long)tok * group)) * P.tokens_q + q_begin + tok;
  };

  // ---- owner rows in registers -----------------------------------------------------------------------------------------------
  const long long orow = o0 + wave * 16 + li;
  const bool ovalid = orow < owners;
  f32x4 r1[NJ], r2[BWD ? NJ : 1];
  {
    const long long r = ovalid ? orow : owners - 1;
    const E* p1 = MODE == GRAD_KV ? key_row(P, P.k, w.seq, k_begin, kvh, (int)r) : q_row(P.q, r);
#pragma unroll
    for (int j = 0; j < NJ; ++j) r1[j] = load4<E>(p1, 16 * j + 4 * g, d, al);
    if (BWD) {
      const E* p2 = MODE == GRAD_KV ? key_row(P, P.v, w.seq, k_begin, kvh, (int)r) : q_row(P.d_out, r);
#pragma unroll
      for (int j = 0; j < NJ; ++j) r2[BWD ? j : 0] = load4<E>(p2, 16 * j + 4 * g, d, al);
    }
  }
  const float sc = P.scale * LOG2E;
  // what an owner row needs: queries: the number of keys they see (and their statistics); keys: the first packed row that sees them
  int limit = 0;
  const long long first_row = MODE == GRAD_KV && P.causal ? max((orow - more) * group, 0LL) : 0;
  float o_lse = 0.f, o_delta = 0.f;
  if (MODE != GRAD_KV) {
    limit = !ovalid ? 0 : P.causal ? min(max(more + 1 + (int)(orow / group), 0), nk) : nk;
    if (MODE == GRAD_Q) {
      if (!SUM_D) {
        const E* po = q_row(P.o, ovalid ? orow : owners - 1);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const f32x4 o = load4<E>(po, 16 * j + 4 * g, d, al);
#pragma unroll
          for (int e = 0; e < 4; ++e) o_delta = __builtin_fmaf(o[e], r2[BWD ? j : 0][e], o_delta);
        }
        o_delta += __shfl_xor(o_delta, 16);
        o_delta += __shfl_xor(o_delta, 32);
      }
      if (ovalid) {
        const long long at = stat_of(orow);
        o_lse = P.lse[at] * LOG2E;
      }
      if (o_lse == -INFINITY) o_lse = INFINITY;  // no weight anywhere
    }
  }

  // ---- the stream ---------------------------------------------------------------------------------------------------------------
  // rows s0 .. s1 - 1: the keys that any owner sees, or the packed query rows that see any owner
  long long s0 = 0, s1 = nk;
  if (MODE == GRAD_KV) {
    s1 = rows;
    if (P.causal) s0 = min(max((o0 - more) * group, 0LL), rows) / BN * BN;
  } else if (P.causal) {
    const long long last = min(o0 + BM, owners) - 1;
    s1 = min(max((long long)more + 1 + last / group, 0LL), (long long)nk);
  }
  if (MODE == FORWARD && P.ranges > 1) {  // this workgroup's range of keys
    const long long per = ((nk + P.ranges - 1) / P.ranges + 63) & ~63;
    s0 = min(blockIdx.z * per, s1);
    s1 = min(s0 + per, s1);
  }
  const int ntiles = (int)((s1 - s0 + BN - 1) / BN);
  constexpr int PIECES = BN * D / 4 / 256;  // 4-channel pieces of a tile per thread
  f32x4 f1[PIECES], f2[PIECES];
  auto fetch = [&](int tile) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = i * 256 + tid;
      const long long r = s0 + (long long)tile * BN + piece / (D / 4);
      const int c = piece % (D / 4) * 4;
      if (r < s1) {
        const E* p1 = MODE == GRAD_KV ? q_row(P.q, r) : key_row(P, P.k, w.seq, k_begin, kvh, (int)r);
        const E* p2 = MODE == GRAD_KV ? q_row(P.d_out, r) : key_row(P, P.v, w.seq, k_begin, kvh, (int)r);
        f1[i] = load4<E>(p1, c, d, al);
        f2[i] = load4<E>(p2, c, d, al);
      } else {
        f1[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        f2[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  };

  constexpr int NACC = MODE == GRAD_KV ? 2 : 1;
  f32x4 acc[NACC][NC][4];  // transposed outputs: lane (i, g) holds channels 64 c + 16 g .. + 15 of owner i: [c][ct][r] is channel 64 c + 16 g + 4 r + ct
#pragma unroll
  for (int x = 0; x < NACC; ++x)
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int ct = 0; ct < 4; ++ct) acc[x][c][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  for (int round = SUM_D ? 0 : 1; round < 2; ++round) {
  float d_sum = 0.f;
  // (past the last tile the half that has none left multiplies zeros)
  if (ntiles > 0) fetch(part);
  // the owner rows are here: left to itself the compiler waits for them in the loop, and with them for the tile just requested
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    asm volatile("" : "+v"(r1[j]));
    if (BWD) asm volatile("" : "+v"(r2[BWD ? j : 0]));
  }
  for (int tile = part; tile - part < ntiles; tile += PARTS) {
    const long long base = s0 + (long long)tile * BN;
    bool odd_value = false;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = i * 256 + tid;
      const int r = piece / (D / 4), c = piece % (D / 4) * 4;
      *reinterpret_cast<f32x4*>(&x1[r][c]) = f1[i];
      *reinterpret_cast<f32x4*>(&x2[r][c]) = f2[i];
      if (MODE == FORWARD) {
#pragma unroll
        for (int e = 0; e < 4; ++e) odd_value = odd_value || !(fabsf(f2[i][e]) < INFINITY);
      }
    }
    if (MODE == GRAD_KV && tid < BN) {
      const long long r = base + tid;
      float a = INFINITY, b = 0.f;
      if (r < s1) {
        const long long at = stat_of(r);
        a = P.lse[at] * LOG2E;
        b = P.delta[at];
        if (a == -INFINITY) a = INFINITY;
      }
      st_lse[MODE == GRAD_KV ? tid : 0] = a;
      st_delta[MODE == GRAD_KV ? tid : 0] = b;
    }
    // a value that is not finite takes the slow way below where not all rows see all keys of the tile
    if (MODE == FORWARD) odd_value = __syncthreads_or(odd_value) != 0;
    else __syncthreads();
    if (tile + PARTS - part < ntiles) fetch(tile + PARTS);

    f32x4 s[2], dp[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
      dp[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(&x1[16 * kb + li][16 * j + 4 * g]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[kb] = mfma(a[e], r1[j][e], s[kb]);
        if (BWD) {
          const f32x4 b = *reinterpret_cast<const f32x4*>(&x2[16 * kb + li][16 * j + 4 * g]);
#pragma unroll
          for (int e = 0; e < 4; ++e) dp[kb] = mfma(b[e], r2[BWD ? j : 0][e], dp[kb]);
        }
      }
    }
    // the tile's rows from .. to - 1 go with the owner row
    int from = 0, to;
    if (MODE == GRAD_KV) {
      from = (int)min(max(first_row - base, 0LL), (long long)BN);
      to = ovalid ? (int)min(s1 - base, (long long)BN) : 0;
    } else {
      to = (int)min(max(min((long long)limit, s1) - base, 0LL), (long long)BN);
    }
    float p[2][4], ds[2][4], keep = 1.f;
    unsigned sees = 0;  // bit 4 kb + r
    if (MODE == FORWARD) {
      float top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool v = 16 * kb + 4 * g + r < to;
          sees |= (unsigned)v << (4 * kb + r);
          s[kb][r] = v ? s[kb][r] * sc : -INFINITY;
          top = fmaxf(top, s[kb][r]);
        }
      top = across_max(top);
      const float m2 = fmaxf(m, top);
      const float ref = m2 == -INFINITY ? 0.f : m2;
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m2;
      float part = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[kb][r] = __builtin_amdgcn_exp2f(s[kb][r] - ref);
          part += p[kb][r];
        }
      l = l * alpha + part;
      keep = alpha;
    } else {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int sr = 16 * kb + 4 * g + r;
          const bool v = sr >= from && sr < to;
          float lse2, delta;
          if (MODE == GRAD_Q) {
            lse2 = o_lse;
            delta = o_delta;
          } else {
            lse2 = st_lse[MODE == GRAD_KV ? sr : 0];
            delta = st_delta[MODE == GRAD_KV ? sr : 0];
          }
          p[kb][r] = v ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], sc, -lse2)) : 0.f;
          ds[kb][r] = v ? p[kb][r] * (dp[kb][r] - delta) : 0.f;
          if (MODE == GRAD_Q) d_sum += ds[kb][r];
        }
      if (MODE == GRAD_Q && round == 0) {
        __syncthreads();
        continue;
      }
    }
    const bool slow = MODE == FORWARD && odd_value && __any(sees != 0xffu);
    // The forward pass sums a tile's products on their own before they join the row's: one chain of additions over thousands of keys
    // loses a digit (float32, 1821 keys: 1.1e-6 of the result, so 4e-7).
    f32x4 sum[NACC][NC][4];
#pragma unroll
    for (int x = 0; x < NACC; ++x)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) sum[x][c][ct] = MODE == FORWARD ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[x][c][ct];
    auto products = [&](auto slow_c) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * kb + 4 * g + r;
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const f32x4 a2 = *reinterpret_cast<const f32x4*>(&x2[row][64 * c + 4 * li]);
            if (decltype(slow_c)::value) {
              // one key at a time, added only to the rows that see it: zero times infinity stays out of the others
#pragma unroll
              for (int gg = 0; gg < 4; ++gg) {
                const bool v = 16 * kb + 4 * gg + r < to;
#pragma unroll
                for (int ct = 0; ct < 4; ++ct) {
                  const f32x4 one = mfma(g == gg ? a2[ct] : 0.f, p[kb][r], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                  for (int e = 0; e < 4; ++e) sum[0][c][ct][e] += v ? one[e] : 0.f;
                }
              }
            } else if (MODE == FORWARD) {
#pragma unroll
              for (int ct = 0; ct < 4; ++ct) sum[0][c][ct] = mfma(a2[ct], p[kb][r], sum[0][c][ct]);
            } else if (MODE == GRAD_Q) {
              const f32x4 a1 = *reinterpret_cast<const f32x4*>(&x1[row][64 * c + 4 * li]);
#pragma unroll
              for (int ct = 0; ct < 4; ++ct) sum[0][c][ct] = mfma(a1[ct], ds[kb][r], sum[0][c][ct]);
            } else {
              const f32x4 a1 = *reinterpret_cast<const f32x4*>(&x1[row][64 * c + 4 * li]);
#pragma unroll
              for (int ct = 0; ct < 4; ++ct) {
                sum[0][c][ct] = mfma(a1[ct], ds[kb][r], sum[0][c][ct]);
                sum[NACC - 1][c][ct] = mfma(a2[ct], p[kb][r], sum[NACC - 1][c][ct]);
              }
            }
          }
        }
    };
    if (slow) products(std::bool_constant<MODE == FORWARD>{});
    else products(std::false_type{});
#pragma unroll
    for (int x = 0; x < NACC; ++x)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) acc[x][c][ct] = MODE == FORWARD ? acc[x][c][ct] * keep + sum[x][c][ct] : sum[x][c][ct];
    __syncthreads();
  }
  if (MODE == GRAD_Q && round == 0) {
    d_sum += __shfl_xor(d_sum, 16);
    d_sum += __shfl_xor(d_sum, 32);
    if (PARTS == 2) {  // both halves' sums
      float* buf = &tiles_lds[0][0][0][0];
      buf[threadIdx.x] = d_sum;
      __syncthreads();
      d_sum += buf[threadIdx.x ^ 256];
      __syncthreads();
    }
    o_delta = d_sum;
  }
  }
  if (MODE == GRAD_Q && ovalid && g == 0 && part == 0) P.delta[stat_of(orow)] = o_delta;

  // ---- epilogue -----------------------------------------------------------------------------------------------------------------
  if (PARTS == 2) {
    // the second half hands over what it has (every wave is past the last barrier of the stream: the tiles are free)
    float* buf = &tiles_lds[0][0][0][0];
    constexpr int REGS = NACC * NC * 16;
    static_assert(PARTS == 1 || (REGS + 2) * 256 <= PARTS * 2 * BN * LS, "a half's sums fit the tiles");
    if (part == 1) {
#pragma unroll
      for (int i = 0; i < REGS; ++i) buf[i * 256 + tid] = acc[i / (NC * 16)][i / 16 % NC][i / 4 % 4][i % 4];
      buf[REGS * 256 + tid] = m;
      buf[(REGS + 1) * 256 + tid] = l;
    }
    __syncthreads();
    if (part == 1) return;
    float a0 = 1.f, a1 = 1.f;
    if (MODE == FORWARD) {
      const float m1 = buf[REGS * 256 + tid], m2 = fmaxf(m, m1), ref = m2 == -INFINITY ? 0.f : m2;
      a0 = __builtin_amdgcn_exp2f(m - ref);
      a1 = __builtin_amdgcn_exp2f(m1 - ref);
      l = l * a0 + buf[(REGS + 1) * 256 + tid] * a1;
      m = m2;
    }
#pragma unroll
    for (int i = 0; i < REGS; ++i) {
      f32x4& x = acc[i / (NC * 16)][i / 16 % NC][i / 4 % 4];
      x[i % 4] = MODE == FORWARD ? x[i % 4] * a0 + buf[i * 256 + tid] * a1 : x[i % 4] + buf[i * 256 + tid];
    }
  }
  float f = P.scale;
  if (MODE == FORWARD) {
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    f = l == 0.f ? 0.f : 1.0f / l;
  }
  if (!ovalid) return;
  if (MODE == FORWARD && P.ranges > 1) {
    const long long at = ((long long)blockIdx.z * P.heads_kv + kvh) * ((long long)P.tokens_q * group) + (long long)q_begin * group + orow;
    if (g == 0) P.part_s[at] = l == 0.f ? -INFINITY : m + __log2f(l);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4*>(P.part_o + at * D + 64 * c + 16 * g + 4 * r) =
            f32x4{acc[0][c][0][r] * f, acc[0][c][1][r] * f, acc[0][c][2][r] * f, acc[0][c][3][r] * f};
    return;
  }
  if (MODE == FORWARD && P.lse != nullptr && g == 0) P.lse[stat_of(orow)] = l == 0.f ? -INFINITY : LN2 * (m + __log2f(l));
  auto target = [&](const Rows<E>& X) -> E* {
    if (MODE == GRAD_KV) return X.p + (k_begin + orow) * X.t + kvh * X.h;
    const int tok = (int)(orow / group);
    return X.p + (long long)(q_begin + tok) * X.t + (kvh * group + (int)(orow - (long long)tok * group)) * X.h;
  };
#pragma unroll
  for (int x = 0; x < NACC; ++x) {
    E* o = target(MODE == FORWARD ? P.out : MODE == GRAD_Q ? P.dq : x == 0 ? P.dk : P.dv);
    const float fx = x == 1 ? 1.0f : f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        store4<E>(o, 64 * c + 16 * g + 4 * r, d, al, acc[x][c][0][r] * fx, acc[x][c][1][r] * fx, acc[x][c][2][r] * fx, acc[x][c][3][r] * fx);
  }
}

template <typename E, int MODE>
hipError_t launch(const SeqParams<E>& P, hipStream_t st) {
  const long long tiles = MODE == GRAD_KV ? tile_bound(P.tokens_k, 1, BM, P.n_seqs) : tile_bound(P.tokens_q, P.group, BM, P.n_seqs);
  if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)tiles, (unsigned)P.heads_kv, (unsigned)(MODE == FORWARD && P.ranges > 1 ? P.ranges : 1));
  auto go = [&](auto dc) -> hipError_t {
    constexpr int D = decltype(dc)::value;
    auto kern = seq_general_kernel<E, D, MODE>;
    // Under a causal mask a launch of up to two workgroups a unit is spread one to a unit (by more LDS than it needs): longest first, two of the
    // longest would share one (us, one / two: 4 prompts of up to 1001 64 / 87, one of 3000 168 / 248; 8 of up to 1001, 900 workgroups 96 / 79;
    // without a mask 113 / 94).
    int pad = 0;
    if (D == 64 && P.causal && (long long)grid.x * grid.y * grid.z <= 2LL * compute_units()) {
      pad = 48 * 1024;
      static std::atomic<unsigned long long> done{0};
      const hipError_t e = allow_lds((const void*)kern, pad, &done);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kern, grid, dim3(256 * parts<D>()), pad, st, P);
    return hipGetLastError();
  };
  if (P.d <= 64) return go(std::integral_constant<int, 64>{});
  if (P.d <= 128) return go(std::integral_constant<int, 128>{});
  return go(std::integral_constant<int, 256>{});
}

}  // namespace

template <typename E>
hipError_t launch_seq_attention_general(const SeqParams<E>& P, hipStream_t st) {
  return launch<E, FORWARD>(P, st);
}
template <typename E>
hipError_t launch_seq_attention_bwd_general(const SeqParams<E>& P, hipStream_t st) {
  if (P.tokens_q > 0) {
    const hipError_t e = launch<E, GRAD_Q>(P, st);
    if (e != hipSuccess) return e;
  }
  return P.tokens_k > 0 ? launch<E, GRAD_KV>(P, st) : hipSuccess;
}

template hipError_t launch_seq_attention_general<float>(const SeqParams<float>&, hipStream_t);
template hipError_t launch_seq_attention_general<bf16_t>(const SeqParams<bf16_t>&, hipStream_t);
template hipError_t launch_seq_attention_bwd_general<float>(const SeqParams<float>&, hipStream_t);
template hipError_t launch_seq_attention_bwd_general<bf16_t>(const SeqParams<bf16_t>&, hipStream_t);

}  // namespace vm
