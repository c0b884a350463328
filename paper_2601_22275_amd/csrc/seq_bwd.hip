// Backward pass of bf16 attention over packed sequences on gfx950: d <= 128, a multiple of 8 (padded to 64 or 128 channels in LDS).
//
// Two launches of one kernel, nothing accumulated across workgroups (the same bits every time):
//   dQ       a workgroup owns packed query rows (token, head of the group) and streams the keys and values they see
//   dK, dV   a workgroup owns keys and streams the packed query rows that see them, of all heads of the group: the sum over the heads
//            that share a key head is part of the product.  Two waves of the workgroup share 32 keys and take every other part of the
//            stream, added at the end in LDS: half the longest chain of work, which is what a launch of few keys and a causal mask (the first
//            keys are seen by all rows) waits for.  Where the keys alone do not fill the card, the rows are cut into ranges as well, whose
//            sums meet in memory and a third launch.
// "Owner" rows (32 per wave) stay in registers as B operands, "stream" rows pass through LDS in tiles, three slots, requested two ahead:
//   G^T = X1 R1^T, dP^T = X2 R2^T       lane (i, g) holds owner row i against 16 of 32 stream rows
//   P = 2^(G scale log2 e - lse log2 e),  dS = P (dP - D)
//   acc^T += Xa^T E                     E = dS or P, converted to bf16 where it stands; Xa^T by LDS transpose reads
// (seven products where five would do with dQ accumulated in memory by atomics.)  The dQ launch leaves {lse log2 e, D} per packed row to the
// other.  D = sum_j P dP is known after the last key only; D' = d_out . out from the stored rows carries the rounding of out, which dP - D does
// not forgive where a row's weight sits on a few keys.  So the launch forms dS' = P (dP - D') and corrects both at the end, with sum_j P = 1:
//   D = D' + sum_j dS'        dq / scale = sum_j dS' k - (sum_j dS') sum_j P k
// at the cost of an eighth product, sum_j P k, on the operands of the first (3 x 4096 tokens forward and backward 652 -> 711 us; D summed in a round of its
// own would be two products).  For dq the sum is of the ROUNDED dS': the weights that the keys really
// get add up to zero, so a row that sits on one key loses no digits to it, nor does what all keys have in common.  Errors of dq and dk stay at 1.2 to
// 1.5 roundings of the result at any sharpness and length (with D' alone 2.7 to 4.4 at logit deviations of 8 and 16): the result's own and that of the
// operands dS and P, which the bf16 matrix units take in eight bits.
// Bound by the matrix units and the LDS reads that feed them (an operand per MFMA): they are busy for 0.50 (dQ) and 0.39 (dK, dV) of the cycles, the vector units for as
// many, and two waves on a SIMD, all that the registers allow, overlap the two only in part.  3 x 4096 causal tokens, 12 heads on 4, d = 128: dQ
// 274 us (883 TFLOP/s of the products issued), dK and dV with their join 340 (710), in single launches under a tracer; forward and backward in a row 679 to
// 717 from card to card.  Operands requested further ahead, G and dP in turn, twice the rows
// between barriers: level, or behind for spilled registers.
#include "seq_device.h"

namespace vm {

namespace {

constexpr int NT = 4;  // 32-row owner tiles of a workgroup
constexpr int NSLOT = 3;

enum { DQ = 0, DKV = 1 };

template <int MODE>
constexpr int waves() {  // two workgroups on a compute unit, or one of twice the waves
  return MODE == DKV ? 2 * NT : NT;
}
template <int D, int MODE>
constexpr int tile_rows() {  // stream rows per LDS tile
  return (D == 128 ? 8 : 16) * waves<MODE>();
}
// k-steps of the second owner tensor that wait in LDS: at d = 128 two sets of accumulators just fill a wave's 256 registers
template <int D>
constexpr int own_in_lds() {
  return D == 128 ? 4 : 0;
}

template <int D, int MODE>
__global__ void __launch_bounds__(64 * waves<MODE>(), 2) seq_bwd_kernel(SeqParams<bf16_t> P) {
  using G = RowGeo<D>;
  constexpr int NW = waves<MODE>();
  constexpr int BK = tile_rows<D, MODE>();
  constexpr int SR = BK;  // floats of a tile's array of statistics
  constexpr int BO = 32 * NT;
  constexpr int SHARE = NW / NT;  // waves on one owner tile
  constexpr int ROW_BYTES = G::ROW_BYTES;
  constexpr int TILE_BYTES = BK * ROW_BYTES;
  constexpr int SLOT_BYTES = 2 * TILE_BYTES;
  constexpr int KS = G::KS, CT = G::CT, CH = G::CH, RPI = G::RPI;
  constexpr int NST = MODE == DKV ? 2 : 0;  // arrays of stream statistics: lse log2 e, D
  constexpr int STATS_OFF = NSLOT * SLOT_BYTES;
  constexpr int STATS_SLOT = NST * SR * 4;
  constexpr int NACC = 2;                  // E = dS, and E = P
  constexpr int NX = MODE == DKV ? 2 : 1;  // dK, dV: their operands are of two tensors (queries, d_out); dQ: of one (keys)
  constexpr bool TIGHT = D == 128;
  constexpr int NG = 2 * KS;
  constexpr int NL = own_in_lds<D>();
  constexpr int OWN_OFF = STATS_OFF + NSLOT * STATS_SLOT;
  auto swz = [](int row) { return G::swz(row); };
  extern __shared__ __attribute__((aligned(16))) char smem[];

  const int kvh = blockIdx.x % P.heads_kv;
  const int tiles = gridDim.x / P.heads_kv, at = blockIdx.x / P.heads_kv;
  // under a causal mask the last queries see most keys, and the first keys are seen by most queries: those start first
  const bool by_work = P.causal && P.n_seqs <= 64;
  const int* own_starts = MODE == DKV ? P.k_starts : P.q_starts;
  const int own_tokens = MODE == DKV ? P.tokens_k : P.tokens_q, per_token = MODE == DKV ? 1 : P.group;
  Span w = by_work ? find_tile_by_work(own_starts, P.n_seqs, own_tokens, per_token, BO, at)
                   : find_tile(own_starts, P.n_seqs, own_tokens, per_token, BO, MODE == DKV ? at : tiles - 1 - at);
  if (MODE == DKV && by_work) w.tile = max((w.count + BO - 1) / BO - 1 - w.tile, 0);
  int q_begin, nq, k_begin, nk;
  if (MODE == DKV) {
    k_begin = w.begin;
    nk = w.count;
    q_begin = start_of(P.q_starts, w.seq, P.tokens_q);
    nq = max(start_of(P.q_starts, w.seq + 1, P.tokens_q) - q_begin, 0);
  } else {
    q_begin = w.begin;
    nq = w.count;
    nk = keys_of(P, w.seq, &k_begin);
  }
  const int group = P.group;
  const int rows = nq * group;  // packed query rows (the host keeps tokens * group below 2^31)
  const int owners = MODE == DKV ? nk : rows;
  const long long first_owner = (long long)w.tile * BO;
  if (first_owner >= owners) return;
  const int o0 = (int)first_owner;
  const int more = nk - nq;  // token i sees keys below more + 1 + i

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ot = wave % NT, part_of = wave / NT;  // owner tile; which part of a stream tile
  const int lane = tid & 63;
  const int ql = lane & 31;
  const int g = lane >> 5;

  // the stream rows lo .. hi - 1 that an owner row sees (or that see it); lo, hi grow with the owner row
  auto range_of = [&](int o, int* lo, int* hi) {
    if (MODE == DKV) {
      *lo = P.causal ? (int)min(max((long long)(o - more) * group, 0LL), (long long)rows) : 0;
      *hi = rows;
    } else {
      *lo = 0;
      *hi = P.causal ? min(max(more + 1 + o / group, 0), nk) : nk;
    }
  };
  const int last_owner = min(o0 + BO, owners) - 1;
  int s0, s1, unused;
  range_of(o0, &s0, &unused);
  range_of(last_owner, &unused, &s1);
  s0 = s0 / 32 * 32;
  if (MODE == DKV && P.ranges > 1) {  // this workgroup's range of rows
    const long long per = ((s1 - s0 + P.ranges - 1) / P.ranges + BK - 1) / BK * BK;
    s0 = (int)min(s0 + blockIdx.y * per, (long long)s1);
    s1 = (int)min(s0 + per, (long long)s1);
  }
  const int ntiles = (s1 - s0 + BK - 1) / BK;

  const bf16_t* qbase = P.q.p + (long long)q_begin * P.q.t + (long long)kvh * group * P.q.h;
  const bf16_t* dobase = P.d_out.p + (long long)q_begin * P.d_out.t + (long long)kvh * group * P.d_out.h;
  const bf16_t* kbase = P.k.p + (long long)k_begin * P.k.t + kvh * P.k.h;
  const bf16_t* vbase = P.v.p + (long long)k_begin * P.v.t + kvh * P.v.h;
  // {lse log2 e, D} of this key head's packed rows
  const long long all_rows = (long long)P.tokens_q * group;
  float* stat_l = P.delta + kvh * all_rows + (long long)q_begin * group;
  float* stat_d = stat_l + P.heads_kv * all_rows;

  // ---- stream tiles: global -> LDS (lanes past the head's channels fetch nothing, their slots are cleared once) -----------------------
  constexpr int NR = BK / (RPI * NW);
  static_assert(BK % (RPI * NW) == 0, "every wave issues the same number of loads per tile");
  const unsigned lds_base = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char*)smem;
  // where the lane's rows of the next tile to request lie: their first row's (token, head), stepped without a division
  int st_tok[MODE == DKV ? NR : 1], st_head[MODE == DKV ? NR : 1];
  const int step_tok = BK / group, step_head = BK - step_tok * group;
  const int last_tok = max(nq - 1, 0);
  auto rewind = [&]() __attribute__((always_inline)) {
    if (MODE == DKV) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int row = s0 + RPI * NW * r + RPI * wave + lane / CH;
        st_tok[r] = row / group;
        st_head[r] = row - st_tok[r] * group;
      }
    }
  };
  auto issue_tile = [&](int t) __attribute__((always_inline)) {
    const unsigned kb = lds_base + (t % NSLOT) * SLOT_BYTES;
    int tid_i = tid;  // the lane's place, derived anew where registers are short
    if (TIGHT) asm volatile("" : "+v"(tid_i));
    const int lane_i = tid_i & 63;
    const int st_row = RPI * wave + lane_i / CH;  // + RPI NW r
    const int st_c = ((lane_i % CH) ^ swz(st_row)) * 8;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const bf16_t *p1, *p2;
      if (MODE == DKV) {
        int tok = st_tok[r], head = st_head[r];
        if (tok > last_tok) {  // rows past the end: copies of the last one, weight zero below
          tok = last_tok;
          head = group - 1;
        }
        p1 = qbase + (long long)tok * P.q.t + head * P.q.h + st_c;
        p2 = dobase + (long long)tok * P.d_out.t + head * P.d_out.h + st_c;
        st_tok[r] += step_tok;
        st_head[r] += step_head;
        if (st_head[r] >= group) {
          st_head[r] -= group;
          ++st_tok[r];
        }
      } else {
        const long long row = min(s0 + t * BK + RPI * NW * r + st_row, nk - 1);
        p1 = kbase + row * P.k.t + st_c;
        p2 = vbase + row * P.v.t + st_c;
      }
      const unsigned dst = __builtin_amdgcn_readfirstlane(kb + (RPI * NW * r + RPI * wave) * ROW_BYTES);
      const unsigned dst2 = dst + TILE_BYTES;
      if (st_c < P.d) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p1), "s"(dst) : "memory", "m0");
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p2), "s"(dst2) : "memory", "m0");
      }
    }
    constexpr int SW = NST * SR / 64;  // waves that fetch statistics, one float per lane
    if (MODE == DKV && wave < SW) {
      const int array = wave / (SR / 64), part = wave % (SR / 64);
      const float* s3 = (array == 0 ? stat_l : stat_d) + min(s0 + t * BK + 64 * part + lane_i, rows - 1);
      const unsigned dst3 = __builtin_amdgcn_readfirstlane(lds_base + STATS_OFF + (t % NSLOT) * STATS_SLOT + wave * 256);
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(s3), "s"(dst3) : "memory", "m0");
    }
  };
  if (P.d < D) {
    const uint4 z = {0u, 0u, 0u, 0u};
    for (int i = tid * 16; i < NSLOT * SLOT_BYTES; i += 64 * NW * 16) *reinterpret_cast<uint4*>(smem + i) = z;
    __syncthreads();
  }
  rewind();
  if (ntiles > 0) issue_tile(0);
  if (ntiles > 1) issue_tile(1);

  // ---- owner rows: B operands in registers -------------------------------------------------------------------------------------------
  const int orow_raw = o0 + ot * 32 + ql;
  const bool ovalid = orow_raw < owners;
  const int orow = ovalid ? orow_raw : owners - 1;
  int lo, hi;
  range_of(orow, &lo, &hi);
  typedef __attribute__((address_space(3))) const bf16x8* lds_b128_ptr;
  typedef __attribute__((address_space(3))) bf16x8* lds_b128_wptr;
  bf16x8 reg1[KS], reg2[KS - NL];
  const unsigned own_base = lds_base + OWN_OFF + (ot * NL * 64 + lane) * 16;  // (written alike by the waves that share it)
  const int otok = MODE == DKV ? 0 : orow / group, ohead = orow - otok * group;
  const bf16x8 zero8 = {0, 0, 0, 0, 0, 0, 0, 0};
  float o_l2 = 0.f, o_delta = 0.f;  // of the owner row where it is a query: lse log2 e, D'
  {
    const bf16_t* op = P.o.p + (long long)(q_begin + otok) * P.o.t + (long long)(kvh * group + ohead) * P.o.h + 8 * g;
    const bf16_t* r1 = MODE == DKV ? kbase + (long long)orow * P.k.t : qbase + (long long)otok * P.q.t + ohead * P.q.h;
    const bf16_t* r2 = MODE == DKV ? vbase + (long long)orow * P.v.t : dobase + (long long)otok * P.d_out.t + ohead * P.d_out.h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bool in = 16 * ks + 8 * g < P.d;
      reg1[ks] = in ? *reinterpret_cast<const bf16x8*>(r1 + 8 * g + 16 * ks) : zero8;
      const bf16x8 x = in ? *reinterpret_cast<const bf16x8*>(r2 + 8 * g + 16 * ks) : zero8;
      if (ks < KS - NL) reg2[ks] = x;
      else *(lds_b128_wptr)(unsigned long long)(own_base + (ks - (KS - NL)) * 1024) = x;
      if (MODE == DQ) {
        const bf16x8 y = in ? *reinterpret_cast<const bf16x8*>(op + 16 * ks) : zero8;
#pragma unroll
        for (int i = 0; i < 8; ++i) o_delta = __builtin_fmaf((float)x[i], (float)y[i], o_delta);
      }
    }
  }
  const float sc2 = P.scale * LOG2E;
  if (MODE == DQ) {
    o_delta += __shfl_xor(o_delta, 32);
    o_l2 = P.lse[(long long)(kvh * group + ohead) * P.tokens_q + q_begin + otok] * LOG2E;
    if (o_l2 == -INFINITY) o_l2 = INFINITY;  // a row that sees nothing: no weight anywhere
  }

  const unsigned a_base = lds_base + ql * ROW_BYTES + ((g ^ swz(ql)) << 4);
  unsigned t_base[2];
  {
    const int rp = lane & 15;
    const int chh = (lane >> 4) & 1;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int row = 8 * hh + 4 * g + (rp >> 2);
      const int lc = 2 * chh + ((rp >> 1) & 1);
      t_base[hh] = lds_base + row * ROW_BYTES + ((lc ^ swz(row)) << 4) + ((rp & 1) << 3);
    }
  }
  typedef __attribute__((address_space(3))) bf16x4* lds_b64_ptr;
  typedef __attribute__((address_space(3))) const f32x4* lds_f32x4_ptr;
  auto rd_row = [&](unsigned addr) __attribute__((always_inline)) -> bf16x8 { return *(lds_b128_ptr)(unsigned long long)addr; };
  auto rd_tr = [&](unsigned a, unsigned b) __attribute__((always_inline)) -> bf16x8 {
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b64_ptr)(unsigned long long)a);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b64_ptr)(unsigned long long)b);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto rd_stat = [&](unsigned addr) __attribute__((always_inline)) -> f32x4 { return *(lds_f32x4_ptr)(unsigned long long)addr; };

  f32x16 acc[NACC][CT];
#pragma unroll
  for (int x = 0; x < NACC; ++x)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][ct][r] = 0.f;
  float d_sum = 0.f, e_sum = 0.f;  // dQ: dS' of the owner row summed before and after its rounding
  constexpr int NOP = NG + 2 * CT * NX;  // operands of a sub-tile: of G, dP, then of the products
  constexpr int PF = TIGHT ? 2 : 3;
  const bool active = o0 + ot * 32 < owners;
  // stream rows that every owner row of the wave goes with lie in whole_lo .. whole_hi - 1
  int whole_lo, whole_hi;
  range_of(min(o0 + ot * 32 + 31, owners - 1), &whole_lo, &unused);
  range_of(min(o0 + ot * 32, owners - 1), &unused, &whole_hi);

  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  bf16x2 ones2;
  ones2[0] = (__bf16)1.0f;
  ones2[1] = (__bf16)1.0f;
  // ---- one 32-row sub-tile of the stream ------------------------------------------------------------------------------------------------
  auto step = [&](unsigned slot, unsigned sslot, auto st_c, int first) __attribute__((always_inline)) {
    constexpr int ST = decltype(st_c)::value;
    constexpr int SUB = ST * 32 * ROW_BYTES;
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) { s[r] = 0.f; dp[r] = 0.f; }
    // operands pass through a ring of four, requested PF ahead and no earlier: left to itself the compiler requests a whole product's at once
    // and spills (opaque copies: address terms are not kept across sub-tiles where registers are short)
    unsigned ab = a_base + slot, tb0 = t_base[0] + slot, tb1 = t_base[1] + slot;
    if (TIGHT) asm volatile("" : "+v"(ab), "+v"(tb0), "+v"(tb1));
    bf16x8 ring[4], own[NL > 0 ? NL : 1];
    auto request = [&](auto ic) __attribute__((always_inline)) {
      constexpr int I = decltype(ic)::value;
      if constexpr (I < KS) {
        ring[I & 3] = rd_row((ab ^ (I << 5)) + SUB);
      } else if constexpr (I < NG) {
        ring[I & 3] = rd_row((ab ^ ((I - KS) << 5)) + SUB + TILE_BYTES);
        if constexpr (I >= NG - NL) own[I - (NG - NL)] = rd_row(own_base + (I - (NG - NL)) * 1024);
      } else if constexpr (I < NOP) {
        constexpr int c = (I - NG) / (CT * NX), ct = (I - NG) / NX % CT, x = (NX - 1) - (I - NG) % NX;  // dV first: P is there before dS
        constexpr int off = SUB + c * 16 * ROW_BYTES + (x == 1 ? TILE_BYTES : 0);
        ring[I & 3] = rd_tr((tb0 ^ (ct << 6)) + off, (tb1 ^ (ct << 6)) + off);
      }
    };
    static_for<0, PF>(request);
    static_for<0, NG>([&](auto ic) __attribute__((always_inline)) {
      constexpr int I = decltype(ic)::value;
      request(std::integral_constant<int, I + PF>{});
      if constexpr (I < KS) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[I & 3], reg1[I], s, 0, 0, 0);
      else if constexpr (I >= NG - NL) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[I & 3], own[I - (NG - NL)], dp, 0, 0, 0);
      else dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[I & 3], reg2[I - KS], dp, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    });
    // register r is stream row first + 8 (r / 4) + 4 g + r % 4
    const bool part = first < whole_lo || first + 32 > whole_hi;
    if (part) {
      // rows that do not go together: a logit of -inf gives no weight, and dP = 0 keeps whatever stood there out of dS
      const int from = lo - first - 4 * g, to = hi - first - 4 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int x = 8 * (r >> 2) + (r & 3);
        const bool v = x >= from && x < to;
        s[r] = v ? s[r] : -INFINITY;
        dp[r] = v ? dp[r] : 0.f;
      }
    }
    bf16x8 pb[2], eb[2];  // P, dS
    f32x4 l2 = {o_l2, o_l2, o_l2, o_l2}, dd = {o_delta, o_delta, o_delta, o_delta};
    auto stats = [&](auto r4_c) __attribute__((always_inline)) {  // of stream rows 8 r4 + 4 g .. + 3
      if (MODE == DKV) {
        const unsigned sa = sslot + (32 * ST + 8 * decltype(r4_c)::value) * 4;
        l2 = rd_stat(sa);
        dd = rd_stat(sa + SR * 4);
      }
    };
    auto score = [&](auto rc) __attribute__((always_inline)) {
      constexpr int r = decltype(rc)::value;
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc2, -l2[r & 3]));
      const float e = p * (dp[r] - dd[r & 3]);
      pb[r >> 3][r & 7] = (__bf16)p;
      eb[r >> 3][r & 7] = (__bf16)e;
      if (MODE == DQ) {
        d_sum += e;
        if constexpr (r & 1) {
          bf16x2 two;
          two[0] = eb[r >> 3][(r & 7) - 1];
          two[1] = eb[r >> 3][r & 7];
          e_sum = __builtin_amdgcn_fdot2_f32_bf16(two, ones2, e_sum, false);
        }
      }
    };
    // The first 16 rows' scores, then the other 16's between the products of the first
    static_for<0, 2>([&](auto r4_c) __attribute__((always_inline)) {
      constexpr int r4 = decltype(r4_c)::value;
      stats(r4_c);
      static_for<4 * r4, 4 * r4 + 4>(score);
      if (TIGHT) __builtin_amdgcn_sched_barrier(0);
    });
    __builtin_amdgcn_sched_barrier(0);
    static_for<NG, NOP>([&](auto ic) __attribute__((always_inline)) {
      constexpr int I = decltype(ic)::value;
      constexpr int c = (I - NG) / (CT * NX), ct = (I - NG) / NX % CT, x = (NX - 1) - (I - NG) % NX;
      request(std::integral_constant<int, I + PF>{});
      if constexpr (MODE == DQ || x == 1) acc[1][ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[I & 3], pb[c], acc[1][ct], 0, 0, 0);
      if constexpr (MODE == DQ || x == 0) acc[0][ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[I & 3], eb[c], acc[0][ct], 0, 0, 0);
      if constexpr (c == 0) {
        constexpr int PER = 8 / (CT * NX), r0 = 8 + PER * (I - NG);
        static_for<r0, r0 + PER>([&](auto rc) __attribute__((always_inline)) {
          if constexpr (decltype(rc)::value % 4 == 0) stats(std::integral_constant<int, decltype(rc)::value / 4>{});
          score(rc);
        });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // Tile t sits in slot t mod 3 and is requested two iterations ahead; the barrier at the top of iteration t publishes it and retires
  // tile t - 1, whose slot tile t + 2 takes.
  for (int t = 0; t < ntiles; ++t) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 2 < ntiles) issue_tile(t + 2);
    if (active) {
      constexpr int MINE = BK / SHARE;  // rows of a tile that are this wave's
      const unsigned slot = (t % NSLOT) * SLOT_BYTES + part_of * (MINE * ROW_BYTES);
      const unsigned sslot = lds_base + STATS_OFF + (t % NSLOT) * STATS_SLOT + 16 * g + part_of * (MINE * 4);
      const int first = s0 + t * BK + part_of * MINE;
      step(slot, sslot, std::integral_constant<int, 0>{}, first);
      if constexpr (MINE == 64) step(slot, sslot, std::integral_constant<int, 1>{}, first + 32);
    }
  }
  if (MODE == DQ) {
    d_sum += __shfl_xor(d_sum, 32);
    e_sum += __shfl_xor(e_sum, 32);
    if (ovalid && g == 0) {
      stat_l[orow] = o_l2;
      stat_d[orow] = o_delta + d_sum;
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[0][ct][r] = __builtin_fmaf(-e_sum, acc[1][ct][r], acc[0][ct][r]);
  }

  __syncthreads();
  int tid_e = threadIdx.x;
  asm volatile("" : "+v"(tid_e));
  const int lane_e = tid_e & 63, ql_e = lane_e & 31, g_e = lane_e >> 5;
  if constexpr (SHARE == 2) {
    // the second wave of an owner tile hands its sums to the first
    typedef __attribute__((address_space(3))) f32x4* lds_f32x4_wptr;
    const unsigned at4 = lds_base + (ot * CT * 4 * 64 + lane_e) * 16;
    static_assert(NT * CT * 4 * 1024 <= OWN_OFF, "one accumulator set of all tiles fits");
#pragma unroll
    for (int x = 0; x < NACC; ++x) {
      if (part_of == 1) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *(lds_f32x4_wptr)(unsigned long long)(at4 + (ct * 4 + c) * 1024) =
                f32x4{acc[x][ct][4 * c], acc[x][ct][4 * c + 1], acc[x][ct][4 * c + 2], acc[x][ct][4 * c + 3]};
      }
      __syncthreads();
      if (part_of == 0) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const f32x4 v = *(lds_f32x4_ptr)(unsigned long long)(at4 + (ct * 4 + c) * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[x][ct][4 * c + e] += v[e];
          }
      }
      __syncthreads();
    }
    if (part_of == 1) return;
  }
  const int row_first = o0 + ot * 32;
  if (MODE == DKV && P.ranges > 1) {
    // [range][dK, dV][key head][token][D]
    if (row_first + ql_e < owners) {
      const long long tokens = (long long)P.heads_kv * P.tokens_k;
#pragma unroll
      for (int x = 0; x < NACC; ++x) {
        float* o = P.part_o + ((2LL * blockIdx.y + x) * tokens + (long long)kvh * P.tokens_k + k_begin + row_first + ql_e) * D + 4 * g_e;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *reinterpret_cast<f32x4*>(o + 32 * ct + 8 * c) = f32x4{acc[x][ct][4 * c], acc[x][ct][4 * c + 1], acc[x][ct][4 * c + 2], acc[x][ct][4 * c + 3]};
      }
    }
    return;
  }

  // ---- epilogue: rows staged in LDS, written as whole lines ------------------------------------------------------------------------------
  char* stage = smem + ot * (32 * ROW_BYTES);
  static_assert(NT * 32 * ROW_BYTES <= NSLOT * SLOT_BYTES, "staged rows fit the tile slots");
#pragma unroll
  for (int x = 0; x < NX; ++x) {
    const float f = x == 1 ? 1.0f : P.scale;
    const Rows<bf16_t>& dst = MODE == DQ ? P.dq : x == 1 ? P.dv : P.dk;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint2 v;
        v.x = pack_bf16(acc[x][ct][4 * c + 0] * f, acc[x][ct][4 * c + 1] * f);
        v.y = pack_bf16(acc[x][ct][4 * c + 2] * f, acc[x][ct][4 * c + 3] * f);
        *reinterpret_cast<uint2*>(stage + ql_e * ROW_BYTES + (((4 * ct + c) ^ swz(ql_e)) << 4) + 8 * g_e) = v;
      }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the staged rows are private to the wave
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int ps = 0; ps < 32 / RPI; ++ps) {
      const int lr = ps * RPI + lane_e / CH;
      const int pc = lane_e % CH;
      const int lc = pc ^ swz(lr);
      const int row = row_first + lr;
      if (row < owners && lc * 8 < P.d) {
        const int tok = MODE == DKV ? row : row / group;
        const long long head = MODE == DKV ? kvh : kvh * group + (row - tok * group);
        bf16_t* o = dst.p + (long long)((MODE == DKV ? k_begin : q_begin) + tok) * dst.t + head * dst.h;
        *reinterpret_cast<uint4*>(o + lc * 8) = *reinterpret_cast<const uint4*>(stage + lr * ROW_BYTES + pc * 16);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Ranges of rows added up: D / 4 lanes per key
template <int D>
__global__ void __launch_bounds__(256) seq_bwd_join_kernel(SeqParams<bf16_t> P) {
  const long long tok = (long long)blockIdx.x * (1024 / D) + threadIdx.x / (D / 4);
  const int kvh = blockIdx.y, x = blockIdx.z, c = threadIdx.x % (D / 4) * 4;
  if (tok >= P.tokens_k || c >= P.d) return;
  if (tok < start_of(P.k_starts, 0, P.tokens_k) || tok >= start_of(P.k_starts, P.n_seqs, P.tokens_k)) return;  // of no sequence
  const long long tokens = (long long)P.heads_kv * P.tokens_k;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < P.ranges; ++r) sum += *reinterpret_cast<const f32x4*>(P.part_o + ((2LL * r + x) * tokens + (long long)kvh * P.tokens_k + tok) * D + c);
  if (x == 0) sum *= P.scale;
  const Rows<bf16_t>& dst = x == 0 ? P.dk : P.dv;
  *reinterpret_cast<uint2*>(dst.p + tok * dst.t + kvh * dst.h + c) = make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
}

template <int D, int MODE>
hipError_t launch(const SeqParams<bf16_t>& P, hipStream_t st) {
  constexpr int LDS = 2 * NSLOT * tile_rows<D, MODE>() * D * 2 + (MODE == DKV ? NSLOT * 2 * tile_rows<D, MODE>() * 4 : 0) + NT * own_in_lds<D>() * 1024;
  const long long tiles = MODE == DKV ? tile_bound(P.tokens_k, 1, 32 * NT, P.n_seqs) : tile_bound(P.tokens_q, P.group, 32 * NT, P.n_seqs);
  if (tiles * P.heads_kv > 0x7fffffffLL) return hipErrorInvalidValue;
  auto kern = seq_bwd_kernel<D, MODE>;
  static std::atomic<unsigned long long> done{0};
  const hipError_t configured = allow_lds((const void*)kern, LDS, &done);
  if (configured != hipSuccess) return configured;
  hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * P.heads_kv), (unsigned)(MODE == DKV && P.ranges > 1 ? P.ranges : 1)), dim3(64 * waves<MODE>()), LDS, st, P);
  hipError_t e = hipGetLastError();
  if (MODE == DKV && P.ranges > 1 && e == hipSuccess) {
    const long long blocks = ((long long)P.tokens_k + 1024 / D - 1) / (1024 / D);
    hipLaunchKernelGGL(seq_bwd_join_kernel<D>, dim3((unsigned)blocks, (unsigned)P.heads_kv, 2), dim3(256), 0, st, P);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// Ranges the rows of queries are cut into for dK and dV: up to three workgroups of 128 keys for every compute unit (which holds one), but none below
// 512 rows of an average sequence.  Forward and backward, us by workgroups a unit, one / two / three / four: 3 x 4096 tokens, 12 heads on 4, d =
// 128 717 / 716 / 683 / 698, without a mask 1255 / 1255 / 1214 / 1209; one sequence of 4096 418 / 414 / 414 / 428; 2 x 2000, 12 heads on 12 202 / 202 /
// 202 / 249; 4 clips of up to 3157 rows on texts of up to 512 keys, 10 heads of 64 108 / 90 / 93 / 93.
int seq_bwd_ranges(int n_seqs, long long tokens_q, long long tokens_k, int heads_kv, int group) {
  const long long blocks = tile_bound(tokens_k, 1, 32 * NT, n_seqs) * heads_kv;
  long long r = 3LL * compute_units() / (blocks > 0 ? blocks : 1);
  const long long most = tokens_q * group / n_seqs / 512;
  if (r > most) r = most;
  return r < 2 ? 1 : r > 32 ? 32 : (int)r;
}

template <int D>
hipError_t launch_seq_bwd_mfma(const SeqParams<bf16_t>& P, hipStream_t st) {
  if (P.tokens_q > 0) {
    const hipError_t e = launch<D, DQ>(P, st);
    if (e != hipSuccess) return e;
  }
  return P.tokens_k > 0 ? launch<D, DKV>(P, st) : hipSuccess;
}

template hipError_t launch_seq_bwd_mfma<64>(const SeqParams<bf16_t>&, hipStream_t);
template hipError_t launch_seq_bwd_mfma<128>(const SeqParams<bf16_t>&, hipStream_t);

}  // namespace vm
