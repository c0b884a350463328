// bf16 attention over packed sequences and over pages on gfx950: d <= 128, a multiple of 8 (padded to 64 or 128 channels in LDS).
//
// One workgroup = 4 waves of 32 query rows, two workgroups on a compute unit; query rows are packed (token, head of the group), so that the heads that share
// keys share a tile and its LDS reads.  Keys and values stream through LDS in tiles (four slots per tensor, loaded two tiles ahead straight
// from memory, chunks swizzled as RowGeo says), and both products are v_mfma_f32_32x32x16_bf16 on transposed operands:
//   S^T = K Q^T        lane (q, g) holds the logits of query q for 16 of 32 keys: sums of a row are per-lane scalars
//   O^T += V^T P^T     A = V^T by LDS transpose reads, B = P^T, the S^T accumulator converted to bf16 where it stands
// p = 2^(s scale log2 e - reference); the reference of a row comes from its first 32 logits and any reference gives the same result (the
// weights have fp32's exponent range in bf16 too): it moves only when a sub-tile's weights add up to more than 2^12, checked after the
// fact (the sub-tile is then formed again).  The accumulators are divided by the sum of the ROUNDED weights, so that a row is an exact convex
// combination; the log-sum-exp is of the unrounded ones.
// The keys that all rows of a workgroup see whole go through a software pipeline over 32-key sub-tiles (logits of n + 1, softmax of n,
// products of n - 1 dealt over the same instruction slots); the tiles at the end of the range that some row sees in part or
// not at all (the diagonal, the ragged end) follow in plain order, with a true running maximum, masks, and a look at the values: zero times
// infinity must not reach a row that does not see the key.
// Bound by the matrix units, with the clock held down by power, where rows are many: 16,384 causal tokens, 12 heads on 4, 763 to 811 us a call at d =
// 128 from card to card (1080 to 1018 TFLOP/s; a large library product reaches 1233; 860 in single launches under a tracer), 433 to 446 at d = 64 (950).  The queries have to be waited for
// in front of the loop: the compiler's own wait for them stood in it and took the tile just requested along (845 us in place of 763 on one card,
// 107 in place of 87 for a frame over pages).  A lone workgroup takes 0.35 us per 32 keys at d = 64, 0.57 at 128, which bounds short prompts (a
// dozen of up to 700 tokens: 17 us).  Level or behind: operands requested up to seven MFMAs ahead instead of three; keys and values requested three
// and two tiles ahead and waited for by count; page addresses kept in scalar registers; two 32-row tiles per wave, which halve the LDS reads and
// leave one wave on a SIMD (16 x 1000 tokens, 12 heads, d = 128: 97 us against 68).
#include <type_traits>

#include "seq_device.h"

namespace vm {

namespace {

constexpr int W2 = 4;  // waves per workgroup
constexpr int NSLOT = 4;
// Sums of a sub-tile's weights above this move the reference (a row has grown by 2^7 and more since it was set): the accumulators then have room
// for values up to 2^(127 - 12 - 17) over 2^17 keys.
constexpr float STEP_LARGE2 = 4096.0f;
constexpr float HEADROOM2 = 16.0f;    // a reference that moves is put this far above the row's maximum
constexpr float MOVE_ALONG2 = 8.0f;   // rows of the wave this far above their reference move along

#define SQ_FENCE() __builtin_amdgcn_sched_barrier(0)
// The hardware does not interlock an MFMA's result against plain vector instructions, and the compiler does not see these MFMAs.  Twelve
// issue slots were measured short (the last register of the last accumulator, copied right behind them, was old); these are twenty-four.
#define SQ_MFMA_RESULT_WAIT() asm volatile("s_nop 15\n\ts_nop 7" ::: "memory")

// BT: key rows of an LDS tile.  32: two workgroups share a compute unit at d = 128, three at d = 64; 64 (d = 64): two, and half the barriers.
template <int D, int BT, bool PAGED, bool SPLIT, bool STAT>
__global__ void __launch_bounds__(64 * W2, 2) seq_attention_kernel(SeqParams<bf16_t> P) {
  using G = RowGeo<D>;
  constexpr int ROW_BYTES = G::ROW_BYTES;
  constexpr int TILE_BYTES = BT * ROW_BYTES;
  constexpr int KS = G::KS, CT = G::CT, CH = G::CH, RPI = G::RPI;
  constexpr int V_OFF = NSLOT * TILE_BYTES;
  constexpr int BQ = 32 * W2;
  auto swz = [](int row) { return G::swz(row); };
  extern __shared__ __attribute__((aligned(16))) char smem[];  // [K|V][NSLOT][BT rows][2 D bytes]
  __shared__ int entry[PAGED ? W2 : 1][64];
  __shared__ RowAt row_at[PAGED ? 2 * W2 : 1][BT];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int ql = lane & 31;
  const int g = lane >> 5;

  // Workgroups with neighbouring numbers go to different XCDs; heads innermost, so that an XCD's share repeats few heads and keeps their
  // keys in its L2.  Later tiles first: under a causal mask they see more keys.
  const int kvh = blockIdx.x % P.heads_kv;
  const int tiles = gridDim.x / P.heads_kv, nth = blockIdx.x / P.heads_kv;
  const Span w = P.causal && P.n_seqs <= 64 ? find_tile_by_work(P.q_starts, P.n_seqs, P.tokens_q, P.group, BQ, nth)
                                            : find_tile(P.q_starts, P.n_seqs, P.tokens_q, P.group, BQ, tiles - 1 - nth);
  const long long rows = (long long)w.count * P.group;
  const long long row_first = (long long)w.tile * BQ;
  if (row_first >= rows) return;
  int k_begin;
  const int nk = keys_of(P, w.seq, &k_begin);
  const int group = P.group;
  const long long more = nk - w.count;  // token i sees keys below more + 1 + i
  // the fewest and the most keys that a row of the workgroup sees
  const long long row_last = min(row_first + BQ, rows) - 1;
  int see_least = nk, see_most = nk;
  if (P.causal) {
    see_least = (int)min(max(more + 1 + row_first / group, 0LL), (long long)nk);
    see_most = (int)min(max(more + 1 + row_last / group, 0LL), (long long)nk);
  }
  int k0 = 0;  // this workgroup's range of keys: k0 .. see_most - 1
  if (SPLIT) {
    const int per = ((nk + P.ranges - 1) / P.ranges + 63) & ~63;
    k0 = min((int)blockIdx.y * per, see_most);
    see_most = min(see_most, k0 + per);
    see_least = max(see_least, k0);
  }
  const int nkeys = see_most - k0;
  const int ntiles = (nkeys + BT - 1) / BT;
  const int nfull = min(max(see_least - k0, 0) / BT, ntiles);  // tiles that every row sees whole

  // ---- global -> LDS ----------------------------------------------------------------------------------------------------------
  // One wave instruction fills 64 consecutive 16-byte slots (RPI rows), each lane fetching the chunk that belongs in its slot.  Lanes whose
  // chunk lies past the head's d channels fetch nothing: their slots are cleared once.  Rows past the last key are copies of it (their
  // weight is zero).  The loads are inline assembly: issued through the builtin, every later LDS read would wait for them.
  constexpr int NR = BT / (RPI * W2);
  static_assert(BT % (RPI * W2) == 0 && (RPI * W2) % 16 == 0, "every wave issues the same number of loads; a lane's rows share a swizzle");
  const int st_row = RPI * wave + lane / CH;  // + RPI W2 r
  const int st_lc = (lane % CH) ^ swz(st_row);
  const bool st_on = st_lc * 8 < P.d;
  const unsigned lds_base = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char*)smem;
  const bf16_t* kbase = P.k.p + kvh * P.k.h + (PAGED ? 0LL : (long long)(k_begin + k0) * P.k.t);
  const bf16_t* vbase = P.v.p + kvh * P.v.h + (PAGED ? 0LL : (long long)(k_begin + k0) * P.v.t);
  // Packed keys: a tile's address is wave-uniform, a lane's place in it a 32-bit offset (the host keeps a tile's rows within 2^31 bytes).
  // Pages: rows lie anywhere.  Their addresses are formed once each: every fourth tile each wave forms those of one of the next four (row_at), from
  // entries of the table that came to LDS four tiles before (entry).  (Sixty-four-bit products in every lane that loads took 9 % of the rate.)
  const int row_k = (int)(2 * P.k.t), row_v = (int)(2 * P.v.t);  // bytes (packed keys)
  const int last_key = max(nk - 1, 0);
  auto key_of = [&](int t) __attribute__((always_inline)) { return min(k0 + t * BT + lane % BT, last_key); };
  auto fetch_entries = [&](int t) __attribute__((always_inline)) {  // past the last tile: the last key's, never used
    const int* e = P.table + w.seq * P.table_stride + key_of(t) / P.page_size;
    const unsigned dst = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long long)(__attribute__((address_space(3))) char*)&entry[wave][0]);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(e), "s"(dst) : "memory", "m0");
  };
  auto prepare_rows = [&](int t) __attribute__((always_inline)) {
    const int e = entry[wave][lane];
    const long long page = e < 0 || e >= P.n_pages ? 0 : e;
    const int slot = key_of(t) % P.page_size;
    row_at[t & 7][lane % BT] = RowAt{kbase + page * P.k.page + slot * P.k.t, vbase + page * P.v.page + slot * P.v.t};
  };
  auto issue_tile = [&](int t) __attribute__((always_inline)) {  // into slot t & 3
    const unsigned kb = lds_base + (t & (NSLOT - 1)) * TILE_BYTES;
    const bf16_t* ktile = kbase + (PAGED ? 0LL : (long long)t * BT * P.k.t);
    const bf16_t* vtile = vbase + (PAGED ? 0LL : (long long)t * BT * P.v.t);
    const int last = nk - 1 - k0 - t * BT;  // the tile's last row that is a key
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int row = RPI * W2 * r + st_row;
      const unsigned dst = __builtin_amdgcn_readfirstlane(kb + (RPI * W2 * r + RPI * wave) * ROW_BYTES);
      const unsigned vdst = dst + V_OFF;
      if (PAGED) {
        const RowAt at = row_at[t & 7][row];
        const bf16_t *ka = at.k + st_lc * 8, *va = at.v + st_lc * 8;
        if (st_on) {
          asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(ka), "s"(dst) : "memory", "m0");
          asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(va), "s"(vdst) : "memory", "m0");
        }
      } else {
        const int at = min(row, last);
        const unsigned ko = at * row_k + st_lc * 16, vo = at * row_v + st_lc * 16;
        if (st_on) {
          asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(ko), "s"(ktile), "s"(dst) : "memory", "m0");
          asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(vo), "s"(vtile), "s"(vdst) : "memory", "m0");
        }
      }
    }
  };
  if (P.d < D) {
    const uint4 z = {0u, 0u, 0u, 0u};
    for (int i = tid * 16; i < 2 * V_OFF; i += 64 * W2 * 16) *reinterpret_cast<uint4*>(smem + i) = z;
    __syncthreads();
  } else {
    // step 0 has no predecessor and multiplies P^T = 0 with slot 3 of V, which may hold anything
    const uint4 z = {0u, 0u, 0u, 0u};
    static_assert(TILE_BYTES % (16 * 64 * W2) == 0, "the clear covers the slot exactly");
#pragma unroll
    for (int r = 0; r < TILE_BYTES / (16 * 64 * W2); ++r) *reinterpret_cast<uint4*>(smem + V_OFF + 3 * TILE_BYTES + (r * 64 * W2 + tid) * 16) = z;
  }
  if (PAGED && ntiles > 0) {
    fetch_entries(wave);  // tiles 0 .. 3
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    prepare_rows(wave);
    fetch_entries(W2 + wave);
    __syncthreads();
  }
  if (ntiles > 0) issue_tile(0);
  if (ntiles > 1) issue_tile(1);

  // ---- queries: B operand of S^T = K Q^T ------------------------------------------------------------------------------------------
  // Packed row r as (token, head), clamped to the last row; and how many keys of this range it sees
  bf16x8 qreg[KS];
  int limit;
  const float sc = P.scale * LOG2E;
  const long long r = min(row_first + wave * 32 + ql, rows - 1);
  const int tok = (int)(r / group);
  const bf16_t* qp = P.q.p + (long long)(w.begin + tok) * P.q.t + (kvh * group + (int)(r - (long long)tok * group)) * P.q.h + 8 * g;
  const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qreg[ks] = 16 * ks + 8 * g < P.d ? *reinterpret_cast<const bf16x8*>(qp + 16 * ks) : zero;
  limit = (P.causal ? (int)min(max(more + 1 + tok, 0LL), (long long)nk) : nk) - k0;

  // ---- LDS read addresses (see RowGeo): everything but these is an instruction immediate --------------------------------------------
  unsigned a_off[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) a_off[ks] = lds_base + ql * ROW_BYTES + (((2 * ks + g) ^ swz(ql)) << 4);
  unsigned t_off[CT][2];
  {
    const int rp = lane & 15;
    const int chh = (lane >> 4) & 1;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int key = 8 * hh + 4 * g + (rp >> 2);
        const int lc = 4 * ct + 2 * chh + ((rp >> 1) & 1);
        t_off[ct][hh] = lds_base + V_OFF + key * ROW_BYTES + ((lc ^ swz(key)) << 4) + ((rp & 1) << 3);
      }
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(a_off[ks]));
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) asm volatile("" : "+v"(t_off[ct][0]), "+v"(t_off[ct][1]));
  typedef __attribute__((address_space(3))) const bf16x8* lds_b128_ptr;
  typedef __attribute__((address_space(3))) bf16x4* lds_b64_ptr;
  auto rd_row = [&](auto kc, int off) __attribute__((always_inline)) -> bf16x8 {
    return *(lds_b128_ptr)(unsigned long long)(a_off[decltype(kc)::value] + off);
  };
  auto rd_tr = [&](unsigned addr) __attribute__((always_inline)) -> bf16x4 {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b64_ptr)(unsigned long long)addr);
  };
  auto rd_value = [&](int ct, int off) __attribute__((always_inline)) -> bf16x8 {
    const bf16x4 lo = rd_tr(t_off[ct][0] + off), hi = rd_tr(t_off[ct][1] + off);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  // ---- the MFMAs, as inline assembly: logits in ordinary registers, products in accumulation registers --------------------------------
  // A vector instruction's result takes two issue slots to reach an MFMA; the plain forms wait for them themselves (the compiler may place copies
  // right in front), the pipeline's operands are older.
  auto mfma_first = [&](f32x16& acc, const bf16x8& a, const bf16x8& b) __attribute__((always_inline)) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "v"(a), "v"(b));
  };
  auto mfma_v = [&](f32x16& acc, const bf16x8& a, const bf16x8& b) __attribute__((always_inline)) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
  };
  auto mfma_a = [&](f32x16& acc, const bf16x8& a, const bf16x8& b) __attribute__((always_inline)) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  };

  auto pipe_first = [&](f32x16& acc, const bf16x8& a, const bf16x8& b) __attribute__((always_inline)) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "v"(a), "v"(b));
  };
  auto pipe_v = [&](f32x16& acc, const bf16x8& a, const bf16x8& b) __attribute__((always_inline)) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
  };
  auto pipe_a = [&](f32x16& acc, const bf16x8& a, const bf16x8& b) __attribute__((always_inline)) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  };

  f32x16 oacc[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[ct][r] = 0.f;
  float msc, ltil, lsum;  // reference, sum of the rounded weights, of the unrounded ones
  msc = NEG_BIG;
  ltil = 0.f;
  lsum = 0.f;

  // ---- one step of the pipeline (see the top): KS groups of logits, then 2 CT groups of products --------
  constexpr int NPV = 2 * CT;
  constexpr int NG = KS + NPV;
  constexpr int PF = 3, RING = 4;
  static_assert(NG % RING == 0 && RING > PF, "ring positions repeat from step to step");
  bf16x8 ring[RING];
  auto request = [&](auto gc, int s_off, int pv_off) __attribute__((always_inline)) {
    constexpr int GI = decltype(gc)::value;
    if constexpr (GI < KS) {
      ring[GI % RING] = rd_row(gc, s_off);
    } else {
      constexpr int c = (GI - KS) / CT, ct = (GI - KS) % CT;
      ring[GI % RING] = rd_value(ct, pv_off + c * 16 * ROW_BYTES);
    }
  };
  auto issue = [&](auto gc, f32x16 &snext, bf16x8 (&pbprev)[2]) __attribute__((always_inline)) {
    constexpr int GI = decltype(gc)::value;
    if constexpr (GI == 0) pipe_first(snext, ring[GI % RING], qreg[GI]);
    else if constexpr (GI < KS) pipe_v(snext, ring[GI % RING], qreg[GI]);
    else pipe_a(oacc[(GI - KS) % CT], ring[GI % RING], pbprev[(GI - KS) / CT]);
  };

  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  bf16x2 ones2;
  ones2[0] = (__bf16)1.0f;
  ones2[1] = (__bf16)1.0f;
  // Two scores of one query tile in three stages, each in an MFMA slot of its own
  float tq[2][2], pq[2][2];
  float ltstep, lstep;
  auto score_scale = [&](auto kc, f32x16 &scur) __attribute__((always_inline)) {
    constexpr int K = decltype(kc)::value, j = K;
    tq[K & 1][0] = __builtin_fmaf(scur[2 * j], sc, -msc);
    tq[K & 1][1] = __builtin_fmaf(scur[2 * j + 1], sc, -msc);
  };
  auto score_exp = [&](auto kc) __attribute__((always_inline)) {
    constexpr int K = decltype(kc)::value;
    pq[K & 1][0] = __builtin_amdgcn_exp2f(tq[K & 1][0]);
    pq[K & 1][1] = __builtin_amdgcn_exp2f(tq[K & 1][1]);
  };
  auto score_sums = [&](auto kc, bf16x8 (&pbcur)[2]) __attribute__((always_inline)) {
    constexpr int K = decltype(kc)::value, j = K;
    bf16x2 pr;
    pr[0] = (__bf16)pq[K & 1][0];
    pr[1] = (__bf16)pq[K & 1][1];
    if (STAT) lstep = (j == 0 ? pq[K & 1][0] : lstep + pq[K & 1][0]) + pq[K & 1][1];
    ltstep = __builtin_amdgcn_fdot2_f32_bf16(pr, ones2, j == 0 ? 0.f : ltstep, false);
    pbcur[j >> 2][2 * (j & 3)] = pr[0];
    pbcur[j >> 2][2 * (j & 3) + 1] = pr[1];
    asm volatile("" : "+v"(ltstep));
    if (STAT) asm volatile("" : "+v"(lstep));
  };
  auto plain_logits = [&](int off, f32x16 &s) __attribute__((always_inline)) {
    static_for<0, KS>([&](auto kc) {
      constexpr int ks = decltype(kc)::value;
      const bf16x8 a = rd_row(kc, off);
      if constexpr (ks == 0) mfma_first(s, a, qreg[ks]);
      else mfma_v(s, a, qreg[ks]);
    });
    SQ_MFMA_RESULT_WAIT();
    SQ_FENCE();
  };
  auto plain_weights = [&](f32x16 &s, bf16x8 (&pb)[2]) __attribute__((always_inline)) {
    static_for<0, 8>([&](auto kc) {
      score_scale(kc, s);
      score_exp(kc);
      score_sums(kc, pb);
    });
    asm volatile("s_nop 1" ::: "memory");
    SQ_FENCE();
  };
  auto plain_products = [&](int off, bf16x8 (&pb)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const bf16x8 a = rd_value(ct, off + c * 16 * ROW_BYTES);
        mfma_a(oacc[ct], a, pb[c]);
      }
  };
  // Products issued so far have reached the accumulators, and nothing reads those before this line
  auto wait_products = [&]() __attribute__((always_inline)) {
    SQ_FENCE();
    SQ_MFMA_RESULT_WAIT();
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) asm volatile("" : "+a"(oacc[ct]));
    SQ_FENCE();
  };
  // Rows whose maximum `cand` has outgrown the reference take one `headroom` above it; what they have is rescaled
  auto move_reference = [&](float cand, float headroom) __attribute__((always_inline)) {
    const float m = cand > msc + MOVE_ALONG2 ? cand + headroom : msc;
    const float alpha = __builtin_amdgcn_exp2f(msc - m);
    lsum *= alpha;
    ltil *= alpha;
    msc = m;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      // one tile at a time, so that the copies out of the accumulation registers do not pile up
      asm volatile("" : "+a"(oacc[ct]));
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[ct][r] *= alpha;
      asm volatile("" : "+a"(oacc[ct]));
      SQ_FENCE();
    }
  };
  auto add_sums = [&]() __attribute__((always_inline)) {
    ltil += ltstep;
    if (STAT) lsum += lstep;
  };
  // S_OFF / PV_OFF: byte offsets (slot and sub-tile) of this step's logits and products; NS_OFF / NPV_OFF: of the next step's
  auto step = [&](auto s_c, auto pv_c, auto ns_c, auto npv_c, f32x16 &scur, f32x16 &snext, bf16x8 (&pbprev)[2],
                  bf16x8 (&pbcur)[2]) __attribute__((always_inline)) {
    constexpr int S_OFF = decltype(s_c)::value, PV_OFF = decltype(pv_c)::value;
    constexpr int NS_OFF = decltype(ns_c)::value, NPV_OFF = decltype(npv_c)::value;
    SQ_FENCE();
    if constexpr (BT == 32) static_for<0, PF>([&](auto gc) { request(gc, S_OFF, PV_OFF); });
    static_for<0, NG>([&](auto gc) {
      constexpr int GI = decltype(gc)::value;
      if constexpr (GI + PF < NG) request(std::integral_constant<int, GI + PF>{}, S_OFF, PV_OFF);
      else if constexpr (BT == 64) request(std::integral_constant<int, GI + PF - NG>{}, NS_OFF, NPV_OFF);
      issue(gc, snext, pbprev);
      static_for<0, 8>([&](auto kc) {
        constexpr int K = decltype(kc)::value;
        constexpr int S0 = K * NG / 8;
        constexpr int S1 = S0 + 1 < NG ? S0 + 1 : NG - 1;
        constexpr int S2 = S0 + 2 < NG ? S0 + 2 : NG - 1;
        if constexpr (S0 == GI) score_scale(kc, scur);
        if constexpr (S1 == GI) score_exp(kc);
        if constexpr (S2 == GI) score_sums(kc, pbcur);
      });
      SQ_FENCE();
    });
    asm volatile("" : "+v"(pbcur[0]), "+v"(pbcur[1]));
    if (__any(ltstep > STEP_LARGE2)) {
      // the sub-tile just finished (its products are not issued yet) is formed again against new references
      f32x16 s;
      plain_logits(NPV_OFF, s);
      move_reference(subtile_max(s) * sc, HEADROOM2);
      plain_logits(NPV_OFF, s);  // again: kept meanwhile they would sit beside the copies of the accumulators
      plain_weights(s, pbcur);
    }
    add_sums();
  };
  const bool active = row_first + wave * 32 < rows;  // a wave of padding only helps to load

  int t = 0;  // tiles done
  auto next_tile = [&](int tt) __attribute__((always_inline)) {
    if (tt > 0) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();  // tile tt + 1 has landed for everyone; everyone is done with tile tt - 2
    }
    if (PAGED && tt % W2 == 0) {
      prepare_rows(tt + W2 + wave);
      fetch_entries(tt + 2 * W2 + wave);
    }
    if (tt + 2 < ntiles) issue_tile(tt + 2);
  };
  // the queries are here: left to itself the compiler waits for them in the loop, and with them for the tile just requested
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qreg[ks]));
  if (ntiles > 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  if (nfull > 0) {
    // Tile t in slot t & 3: during tile t the products of tile t - 1's last sub-tile are outstanding, tile t + 1 is resident (its first
    // logits are needed a step ahead; behind the last whole tile they are of what comes there, and dropped), t + 2 in flight.
    f32x16 sA, sB;
    bf16x8 pbA[2], pbB[2];
    const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < 2; ++c) pbB[c] = zero;
    if (active) {
      plain_logits(0, sA);
      msc = fmaxf(subtile_max(sA) * sc, NEG_BIG);
      if constexpr (BT == 64) static_for<0, PF>([&](auto gc) { request(gc, 32 * ROW_BYTES, 3 * TILE_BYTES + 32 * ROW_BYTES); });
    }
    auto tile_iteration = [&](auto slot_c, int tt) __attribute__((always_inline)) {
      constexpr int SLOT = decltype(slot_c)::value;
      next_tile(tt);
      constexpr int kp = ((SLOT + 3) & 3) * TILE_BYTES;
      constexpr int kt = SLOT * TILE_BYTES;
      constexpr int kn = ((SLOT + 1) & 3) * TILE_BYTES;
      constexpr int HALF = 32 * ROW_BYTES;
      if (active && BT == 32) {
        constexpr int k2 = ((SLOT + 2) & 3) * TILE_BYTES;
        step(std::integral_constant<int, kn>{}, std::integral_constant<int, kp>{}, std::integral_constant<int, k2>{},
             std::integral_constant<int, kt>{}, SLOT % 2 ? sB : sA, SLOT % 2 ? sA : sB, SLOT % 2 ? pbA : pbB, SLOT % 2 ? pbB : pbA);
      } else if (active) {
        step(std::integral_constant<int, kt + HALF>{}, std::integral_constant<int, kp + HALF>{}, std::integral_constant<int, kn>{},
             std::integral_constant<int, kt>{}, sA, sB, pbB, pbA);
        step(std::integral_constant<int, kn>{}, std::integral_constant<int, kt>{}, std::integral_constant<int, kn + HALF>{},
             std::integral_constant<int, kt + HALF>{}, sB, sA, pbA, pbB);
      }
    };
    for (int t0 = 0; t0 < nfull; t0 += 4) {  // four tiles per trip: slot offsets are immediates
      tile_iteration(std::integral_constant<int, 0>{}, t0);
      if (t0 + 1 < nfull) tile_iteration(std::integral_constant<int, 1>{}, t0 + 1);
      if (t0 + 2 < nfull) tile_iteration(std::integral_constant<int, 2>{}, t0 + 2);
      if (t0 + 3 < nfull) tile_iteration(std::integral_constant<int, 3>{}, t0 + 3);
    }
    t = nfull;
    if (active) {
      // the products of the last sub-tile; with one sub-tile per tile its weights' set goes by the slot
      if (BT == 32 && (nfull & 1)) {
        pbB[0] = pbA[0];
        pbB[1] = pbA[1];
        asm volatile("s_nop 1" ::: "memory");
      }
      plain_products(((nfull - 1) & 3) * TILE_BYTES + (BT - 32) * ROW_BYTES, pbB);
      wait_products();
    }
  }

  // ---- tiles that some row sees in part -------------------------------------------------------------------------------------------
  // what the wave's first and last row see of the range
  const int wave_least = min(__builtin_amdgcn_readfirstlane(limit), nkeys), wave_most = min(__builtin_amdgcn_readfirstlane(__shfl(limit, 31)), nkeys);
  for (; t < ntiles; ++t) {
    next_tile(t);
    if (!active) continue;
#pragma unroll 1
    for (int sub = 0; sub < BT / 32; ++sub) {
      const int off = (t & 3) * TILE_BYTES + sub * 32 * ROW_BYTES;
      const int first = t * BT + 32 * sub;
      if (first >= wave_most) break;
      const bool part = first + 32 > wave_least;
      const bool odd = part && odd_values<ROW_BYTES>(lds_base + V_OFF + off);
      f32x16 s;
      bf16x8 pb[2];
      plain_logits(off, s);
      if (part) {
        const int left = min(limit, nkeys) - first - 4 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < left ? s[r] : -INFINITY;
      }
      const float top = subtile_max(s) * sc;
      if (__any(top > msc + MOVE_ALONG2)) move_reference(top, 0.f);
      plain_weights(s, pb);
      add_sums();
      if (!odd) {
        plain_products(off, pb);
        wait_products();
        continue;
      }
      // a value that is not finite: one key at a time, added to the rows that see it
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {
          const int e = ((i >> 3) & 1) * 4 + (i & 3), half = (i >> 2) & 1;  // key 16 c + 8 (e / 4) + 4 half + e % 4 = 16 c + i
          const uint32_t part = half == g ? (e & 1 ? 0xffff0000u : 0xffffu) : 0u;  // that key's element alone, in 32-bit word e / 2
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            uint32_t a32[4];
            bf16x8 a = rd_value(ct, off + c * 16 * ROW_BYTES);
            __builtin_memcpy(a32, &a, 16);
#pragma unroll
            for (int x = 0; x < 4; ++x) a32[x] &= x == e >> 1 ? part : 0u;
            __builtin_memcpy(&a, a32, 16);
            const bool v = first + 16 * c + i < min(limit, nkeys);
            f32x16 one;
            mfma_first(one, a, pb[c]);
            SQ_MFMA_RESULT_WAIT();
            SQ_FENCE();
            asm volatile("" : "+a"(oacc[ct]));
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[ct][r] += v ? one[r] : 0.f;
            asm volatile("" : "+a"(oacc[ct]));
            SQ_FENCE();
          }
        }
    }
  }
  // ---- epilogue: normalised rows, staged in LDS, leave as whole rows ------------------------------------------------------------------
  __syncthreads();
  int tid_e = threadIdx.x;
  asm volatile("" : "+v"(tid_e));
  const int lane_e = tid_e & 63, ql_e = lane_e & 31, g_e = lane_e >> 5;
  const long long wave_first = row_first + wave * 32;
  char* stage = smem + wave * (32 * ROW_BYTES);
  static_assert(W2 * 32 * ROW_BYTES <= 2 * V_OFF, "staged rows fit the slots");
  SQ_FENCE();
  const long long orow = wave_first + ql_e;
  const float lt = ltil + __shfl_xor(ltil, 32);
  const float inv = lt == 0.f ? 0.f : 1.0f / lt;
  if (SPLIT) {
    if (orow < rows) {
      // partial result of this range: [range][key head][packed row of all sequences]
      const long long at = ((long long)blockIdx.y * P.heads_kv + kvh) * ((long long)P.tokens_q * group) + (long long)w.begin * group + orow;
      if (g_e == 0) P.part_s[at] = lt == 0.f ? -INFINITY : msc + __log2f(lt);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x4 x = {oacc[ct][4 * c + 0] * inv, oacc[ct][4 * c + 1] * inv, oacc[ct][4 * c + 2] * inv, oacc[ct][4 * c + 3] * inv};
          *reinterpret_cast<f32x4*>(P.part_o + at * D + 32 * ct + 8 * c + 4 * g_e) = x;
        }
    }
    return;
  }
  if (STAT) {
    const float l = lsum + __shfl_xor(lsum, 32);
    if (orow < rows && g_e == 0) {
      const int tok = (int)(orow / group);
      P.lse[(long long)(kvh * group + (int)(orow - (long long)tok * group)) * P.tokens_q + w.begin + tok] = l == 0.f ? -INFINITY : LN2 * (msc + __log2f(l));
    }
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint2 x;
      x.x = pack_bf16(oacc[ct][4 * c + 0] * inv, oacc[ct][4 * c + 1] * inv);
      x.y = pack_bf16(oacc[ct][4 * c + 2] * inv, oacc[ct][4 * c + 3] * inv);
      *reinterpret_cast<uint2*>(stage + ql_e * ROW_BYTES + (((4 * ct + c) ^ swz(ql_e)) << 4) + 8 * g_e) = x;
    }
  if (!SPLIT) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the staged rows are private to the wave
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int ps = 0; ps < 32 / RPI; ++ps) {
      const int lr = ps * RPI + lane_e / CH;
      const int pc = lane_e % CH;
      const int lc = pc ^ swz(lr);
      const long long r = wave_first + lr;
      if (r < rows && lc * 8 < P.d) {
        const int tok = (int)(r / group);
        bf16_t* o = P.out.p + (long long)(w.begin + tok) * P.out.t + (kvh * group + (int)(r - (long long)tok * group)) * P.out.h;
        *reinterpret_cast<uint4*>(o + lc * 8) = *reinterpret_cast<const uint4*>(stage + lr * ROW_BYTES + pc * 16);
      }
    }
  }
}

template <int D, int BT, bool PAGED, bool SPLIT, bool STAT>
hipError_t launch(const SeqParams<bf16_t>& P, hipStream_t st) {
  constexpr int LDS = 2 * NSLOT * BT * D * 2;
  const long long blocks = tile_bound(P.tokens_q, P.group, 32 * W2, P.n_seqs) * P.heads_kv;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  auto kern = seq_attention_kernel<D, BT, PAGED, SPLIT, STAT>;
  static std::atomic<unsigned long long> done{0};
  const hipError_t configured = allow_lds((const void*)kern, LDS, &done);
  if (configured != hipSuccess) return configured;
  hipLaunchKernelGGL(kern, dim3((unsigned)blocks, (unsigned)(SPLIT ? P.ranges : 1)), dim3(64 * W2), LDS, st, P);
  return hipGetLastError();
}

#undef SQ_FENCE
#undef SQ_MFMA_RESULT_WAIT

}  // namespace

template <int D>
hipError_t launch_seq_attention_mfma(const SeqParams<bf16_t>& P, hipStream_t st) {
  auto run = [&](auto bt) -> hipError_t {
    constexpr int BT = decltype(bt)::value;
    if (P.page_size > 0) return launch<D, BT, true, false, false>(P, st);
    return P.lse != nullptr ? launch<D, BT, false, false, true>(P, st) : launch<D, BT, false, false, false>(P, st);
  };
  using rows32 = std::integral_constant<int, 32>;
  using rows64 = std::integral_constant<int, 64>;
  if constexpr (D == 64) {
    // Tiles of 64 keys while two workgroups a unit take the whole launch, tiles of 32 and three of them beyond (64 / 32, us: a dozen prompts of up to 700
    // tokens, 12 heads on 4, 440 workgroups 19.1 / 20.0; 40 of them 39.8 / 33.4; 4 clips on 512 keys, 10 heads, 670 23.2 / 17.8; 16,384 causal tokens,
    // 12 heads, 1536 454 / 446, 8192 without a mask 231 / 225).
    if (P.page_size > 0 && P.ranges > 1) return launch<D, 64, true, true, false>(P, st);
    return tile_bound(P.tokens_q, P.group, 32 * W2, P.n_seqs) * P.heads_kv > 2LL * compute_units() ? run(rows32{}) : run(rows64{});
  } else {
    if (P.page_size > 0 && P.ranges > 1) return launch<D, 32, true, true, false>(P, st);
    return run(rows32{});
  }
}

// This file is compiled once per head dimension.
template hipError_t launch_seq_attention_mfma<VM_SEQ_D>(const SeqParams<bf16_t>&, hipStream_t);

}  // namespace vm
