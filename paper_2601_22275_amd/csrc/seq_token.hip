// bf16 attention of few query rows over long caches on gfx950 (single tokens, short chunks; d <= 128, a multiple of 8), and the join of
// ranges of keys.
//
//   out = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m)     is the same sum over ranges of keys once each carries its own m.
// The cache is read once and bounds the kernel (8 TB/s); up to 32 packed rows (token, head of the group) share that read.  A workgroup is two
// waves that take 32-key sub-tiles of its range in turn, each with LDS slots, a running maximum, a sum and accumulators of its own: no
// barrier in the loop, a wave waits for its own loads only; two workgroups share a compute unit, so that one's start and end pass behind the
// other's stream.  The waves join through LDS at the end, the ranges (blockIdx.y) through memory and a second launch.
// 16 single tokens over up to 16,384 keys, 40 heads on 8, d = 128 (585 MB): 130 us, 4.5 TB/s with the join, where a large copy moves 5.0;
// four waves in one workgroup 4 % more, every lane forming the addresses of the rows it loads 17 %, queries waited for in the loop 3 %.  d = 64, 40 heads on 10 (366 MB): 95 us,
// 3.9 TB/s; with four sub-tiles in LDS and two workgroups on a unit 110.  Products as in seq_mfma.hip: S^T = K Q^T and O^T += V^T P^T, both
// v_mfma_f32_32x32x16_bf16.
#include "seq_device.h"

namespace vm {

namespace {

constexpr int NW = 2;

constexpr int NS = 2;  // sub-tiles in LDS per wave: 64 KB a workgroup at d = 128, half that at d = 64 (two and four workgroups on a unit)

template <int D>
__global__ void __launch_bounds__(64 * NW, D == 64 ? 3 : 2) seq_token_kernel(SeqParams<bf16_t> P) {
  using G = RowGeo<D>;
  constexpr int ROW_BYTES = G::ROW_BYTES, KS = G::KS, CT = G::CT, CH = G::CH, RPI = G::RPI;
  constexpr int SUB_BYTES = 32 * ROW_BYTES;
  constexpr int NR = 32 / RPI;               // loads of a tensor per sub-tile
  constexpr int SLOT_BYTES = 2 * SUB_BYTES;  // keys, then values
  constexpr int BQ = 32;
  auto swz = [](int row) { return G::swz(row); };
  extern __shared__ __attribute__((aligned(16))) char smem[];  // [wave][NS][K|V][32 rows]
  __shared__ float wave_m[NW][32], wave_l[NW][32];
  __shared__ int pages[NW][2 * NS][64];  // entries of the table
  __shared__ RowAt row_at[NW][32];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ql = lane & 31, g = lane >> 5;
  const int tiles = gridDim.x / P.heads_kv;
  const int kvh = blockIdx.x / tiles;
  const Span w = find_tile(P.q_starts, P.n_seqs, P.tokens_q, P.group, BQ, blockIdx.x - kvh * tiles);
  const long long rows = (long long)w.count * P.group;
  const long long row_first = (long long)w.tile * BQ;
  if (row_first >= rows) return;
  int unused;
  const int nk = keys_of(P, w.seq, &unused);
  const int group = P.group;
  const long long more = nk - w.count;
  const long long row_last = min(row_first + BQ, rows) - 1;
  int see_most = nk;
  if (P.causal) see_most = (int)min(max(more + 1 + row_last / group, 0LL), (long long)nk);
  int k0 = 0;
  if (P.ranges > 1) {
    const int per = ((nk + P.ranges - 1) / P.ranges + 63) & ~63;
    k0 = min((int)blockIdx.y * per, see_most);
    see_most = min(see_most, k0 + per);
  }
  const int nsub = (see_most - k0 + 31) / 32;  // sub-tiles; this wave's: wave, wave + NW, ...
  const int mine = nsub > wave ? (nsub - wave + NW - 1) / NW : 0;

  // ---- global -> LDS, wave by wave ------------------------------------------------------------------------------------------------
  const unsigned lds_base = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char*)smem + wave * (NS * SLOT_BYTES);
  const bf16_t* kbase = P.k.p + kvh * P.k.h;
  const bf16_t* vbase = P.v.p + kvh * P.v.h;
  // Lane i % 32 looks after key i of a sub-tile.  Its entry of the table goes to LDS the same way, ahead of the sub-tile's rows by NS sub-tiles
  // and in front of a sub-tile's own loads: the wait for those is the wait for it.  (An ordinary load of it would be waited for with
  // everything behind it.)
  const int last_key = max(nk - 1, 0);
  const unsigned ring = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char*)&pages[wave][0][0];
  auto key_of = [&](int i) { return min(k0 + 32 * (wave + NW * i) + ql, last_key); };
  auto fetch_page = [&](int i) {
    const int* entry = P.table + w.seq * P.table_stride + key_of(i) / P.page_size;
    const unsigned dst = __builtin_amdgcn_readfirstlane(ring + (i % (2 * NS)) * 256);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(entry), "s"(dst) : "memory", "m0");
  };
  // The rows' addresses, formed once each, pass through LDS to the lanes that load them
  auto prepare = [&](int i) {
    const int p = pages[wave][i % (2 * NS)][lane];
    const long long page = p < 0 || p >= P.n_pages ? 0 : p;
    const int slot = key_of(i) % P.page_size;
    row_at[wave][ql] = RowAt{kbase + page * P.k.page + slot * P.k.t, vbase + page * P.v.page + slot * P.v.t};  // (both halves of the wave alike)
  };
  auto issue = [&](int i) {
    fetch_page(i + NS);  // (past the last sub-tile: the last key's, never used)
    const unsigned base = lds_base + (i % NS) * SLOT_BYTES;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int row = RPI * r + lane / CH;
      const int c = ((lane % CH) ^ swz(row)) * 8;
      const RowAt at = row_at[wave][row];
      const bf16_t *ka = at.k + c, *va = at.v + c;
      const unsigned dst = __builtin_amdgcn_readfirstlane(base + RPI * r * ROW_BYTES);
      const unsigned vdst = dst + SUB_BYTES;
      if (c < P.d) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(ka), "s"(dst) : "memory", "m0");
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(va), "s"(vdst) : "memory", "m0");
      }
    }
  };
  if (P.d < D) {  // chunks past the head's channels are never loaded
    const uint4 z = {0u, 0u, 0u, 0u};
    for (int i = tid * 16; i < NW * NS * SLOT_BYTES; i += 64 * NW * 16) *reinterpret_cast<uint4*>(smem + i) = z;
    __syncthreads();
  }
  if (mine > 0) {
#pragma unroll 1
    for (int i = 0; i < NS; ++i) fetch_page(i);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int i = 0; i < min(NS, mine); ++i) {
      prepare(i);
      issue(i);
    }
  }

  // ---- queries ----------------------------------------------------------------------------------------------------------------------
  bf16x8 qreg[KS];
  int limit;
  const float sc = P.scale * LOG2E;
  {
    const long long r = min(row_first + ql, rows - 1);
    const int tok = (int)(r / group);
    const bf16_t* qp = P.q.p + (long long)(w.begin + tok) * P.q.t + (kvh * group + (int)(r - (long long)tok * group)) * P.q.h + 8 * g;
    const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qreg[ks] = 16 * ks + 8 * g < P.d ? *reinterpret_cast<const bf16x8*>(qp + 16 * ks) : zero;
    limit = min(P.causal ? (int)min(max(more + 1 + tok, 0LL), (long long)nk) : nk, see_most);
    // the queries are here: left to itself the compiler waits for them in the loop, and with them for the sub-tiles under way
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qreg[ks]));
  }

  typedef __attribute__((address_space(3))) const bf16x8* lds_b128_ptr;
  typedef __attribute__((address_space(3))) bf16x4* lds_b64_ptr;
  unsigned a_base = lds_base + ql * ROW_BYTES + ((g ^ swz(ql)) << 4);  // row reads: chunk 2 ks + g
  unsigned t_base[2];                                                  // transpose reads of the values
  {
    const int rp = lane & 15;
    const int chh = (lane >> 4) & 1;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int key = 8 * hh + 4 * g + (rp >> 2);
      const int lc = 2 * chh + ((rp >> 1) & 1);
      t_base[hh] = lds_base + SUB_BYTES + key * ROW_BYTES + ((lc ^ swz(key)) << 4) + ((rp & 1) << 3);
    }
  }
  f32x16 acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[ct][r] = 0.f;
  float m = NEG_BIG, l = 0.f;
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  bf16x2 ones2;
  ones2[0] = (__bf16)1.0f;
  ones2[1] = (__bf16)1.0f;

#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    // this sub-tile's loads have arrived when no more than those of the one behind it are under way
    constexpr int LOADS = 2 * NR + 1;
    if (i + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (i + NS < mine) prepare(i + NS);  // (its pages came in front of this sub-tile's rows)
    const unsigned off = (i % NS) * SLOT_BYTES;
    const int first = k0 + 32 * (wave + NW * i);
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 a = *(lds_b128_ptr)(unsigned long long)((a_base ^ (ks << 5)) + off);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[ks], s, 0, 0, 0);
    }
    const int left = limit - first - 4 * g;  // register r is key 8 (r / 4) + 4 g + r % 4
    const bool part = __any(limit < first + 32);
    if (part) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < left ? s[r] : -INFINITY;
    }
    // The reference moves where a row's maximum has outgrown it by 2^8 (any reference gives the same result), and for all rows of the wave
    const float top = subtile_max(s) * sc;
    if (__any(top > m + 8.0f)) {
      const float m2 = fmaxf(m, top);
      const float alpha = __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[ct][r] *= alpha;
    }
    bf16x8 pb[2];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      bf16x2 pr;
      pr[0] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -m));
      pr[1] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], sc, -m));
      l = __builtin_amdgcn_fdot2_f32_bf16(pr, ones2, l, false);  // of the rounded weights: rows are exact convex combinations
      pb[r >> 3][r & 7] = pr[0];
      pb[r >> 3][(r & 7) + 1] = pr[1];
    }
    auto value = [&](int c, int ct) -> bf16x8 {
      const unsigned at = off + c * 16 * ROW_BYTES;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b64_ptr)(unsigned long long)((t_base[0] ^ (ct << 6)) + at));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b64_ptr)(unsigned long long)((t_base[1] ^ (ct << 6)) + at));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    if (!part || !odd_values<ROW_BYTES>(lds_base + SUB_BYTES + off)) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) acc[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(c, ct), pb[c], acc[ct], 0, 0, 0);
    } else {
      // a value that is not finite: one key at a time, added to the rows that see it (zero times infinity stays out of the others)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll 1
        for (int k = 0; k < 16; ++k) {
          const int e = ((k >> 3) & 1) * 4 + (k & 3), half = (k >> 2) & 1;
          const uint32_t one_key = half == g ? (e & 1 ? 0xffff0000u : 0xffffu) : 0u;
          const bool v = first + 16 * c + k < limit;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            uint32_t a32[4];
            bf16x8 a = value(c, ct);
            __builtin_memcpy(a32, &a, 16);
#pragma unroll
            for (int x = 0; x < 4; ++x) a32[x] &= x == e >> 1 ? one_key : 0u;
            __builtin_memcpy(&a, a32, 16);
            f32x16 one;
#pragma unroll
            for (int r = 0; r < 16; ++r) one[r] = 0.f;
            one = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[c], one, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[ct][r] += v ? one[r] : 0.f;
          }
        }
    }
    if (i + NS < mine) {
      // the slot's reads are done (their results went into the products above) before it is filled again
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      issue(i + NS);
    }
  }

  // ---- the waves join -----------------------------------------------------------------------------------------------------------------
  l += __shfl_xor(l, 32);
  if (g == 0) {
    wave_m[wave][ql] = m;
    wave_l[wave][ql] = l;
  }
  __syncthreads();  // every wave is done with its slots, too
  float top = NEG_BIG, total = 0.f;
#pragma unroll
  for (int x = 0; x < NW; ++x) top = fmaxf(top, wave_m[x][ql]);
#pragma unroll
  for (int x = 0; x < NW; ++x) total += wave_l[x][ql] * __builtin_amdgcn_exp2f(wave_m[x][ql] - top);
  const float f = total == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top) / total;
  // [wave][32 rows][D + 4] floats: 16-byte pieces of consecutive rows on different banks
  constexpr int LS = D + 4;
  static_assert(NW * 32 * LS * 4 <= NW * NS * SLOT_BYTES, "the partial rows fit the slots");
  float* stage = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<f32x4*>(stage + (wave * 32 + ql) * LS + 32 * ct + 8 * c + 4 * g) =
          f32x4{acc[ct][4 * c] * f, acc[ct][4 * c + 1] * f, acc[ct][4 * c + 2] * f, acc[ct][4 * c + 3] * f};
  const long long part_row = ((long long)blockIdx.y * P.heads_kv + kvh) * ((long long)P.tokens_q * group) + (long long)w.begin * group + row_first;
  if (P.ranges > 1 && wave == 0 && g == 0 && row_first + ql < rows) P.part_s[part_row + ql] = total == 0.f ? -INFINITY : top + __log2f(total);
  __syncthreads();
  for (int i = tid; i < 32 * (D / 4); i += 64 * NW) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    const long long r = row_first + row;
    if (r >= rows) break;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < NW; ++y) x += *reinterpret_cast<const f32x4*>(stage + (y * 32 + row) * LS + c);
    if (P.ranges > 1) {
      *reinterpret_cast<f32x4*>(P.part_o + (part_row + row) * D + c) = x;
    } else if (c < P.d) {
      const int tok = (int)(r / group);
      bf16_t* o = P.out.p + (long long)(w.begin + tok) * P.out.t + (kvh * group + (int)(r - (long long)tok * group)) * P.out.h;
      uint2 y;
      y.x = pack_bf16(x[0], x[1]);
      y.y = pack_bf16(x[2], x[3]);
      *reinterpret_cast<uint2*>(o + c) = y;
    }
  }
}

// Ranges of keys joined: a row's partial results weigh 2^(their log-sum) relative to the largest.  D / 4 lanes take a packed row's channels; where
// ranges are many, GROUPS such groups share the row and its ranges (one group after another's load, 64 ranges took 60 us).
template <typename E, int D, int GROUPS>
__global__ void __launch_bounds__(256) seq_join_kernel(SeqParams<E> P) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / GROUPS;
  static_assert(ROWS >= 1, "a workgroup holds a row's groups");
  __shared__ f32x4 sums[GROUPS > 1 ? GROUPS : 1][ROWS][LANES];
  __shared__ float totals[GROUPS > 1 ? GROUPS : 1][ROWS];
  const int lane = threadIdx.x % LANES, local = threadIdx.x / LANES % ROWS, grp = threadIdx.x / LANES / ROWS;
  const long long all = (long long)P.tokens_q * P.group;  // packed rows of a key head
  const long long row = (long long)blockIdx.x * ROWS + local;
  const int kvh = blockIdx.y, c = lane * 4;
  const int tok = (int)(min(row, all - 1) / P.group);
  const bool in = row < all && tok >= start_of(P.q_starts, 0, P.tokens_q) && tok < start_of(P.q_starts, P.n_seqs, P.tokens_q);  // of a sequence
  const long long step = P.heads_kv * all, at = kvh * all + row;
  float top = NEG_BIG, total = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (in) {
#pragma unroll 4
    for (int x = 0; x < P.ranges; ++x) top = fmaxf(top, P.part_s[x * step + at]);
    // (a range of which the row sees nothing has left zeros and a log-sum of -inf)
#pragma unroll 4
    for (int x = grp; x < P.ranges; x += GROUPS) {
      const float f = __builtin_amdgcn_exp2f(P.part_s[x * step + at] - top);
      total += f;
      o += *reinterpret_cast<const f32x4*>(P.part_o + (x * step + at) * D + c) * f;
    }
  }
  if (GROUPS > 1) {
    sums[grp][local][lane] = o;
    if (lane == 0) totals[grp][local] = total;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int x = 1; x < GROUPS; ++x) {
      o += sums[x][local][lane];
      total += totals[x][local];
    }
  }
  if (!in || c >= P.d) return;
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  E* out = P.out.p + (long long)tok * P.out.t + (kvh * P.group + (int)(row - (long long)tok * P.group)) * P.out.h + c;
  if (P.aligned) {
    if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    else *reinterpret_cast<f32x4*>(out) = o * inv;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < P.d) store_f<E>(out + e, o[e] * inv);
  }
}

}  // namespace

template <int D>
hipError_t launch_seq_token(const SeqParams<bf16_t>& P, hipStream_t st) {
  constexpr int LDS = NW * NS * 2 * 32 * D * 2;
  const long long blocks = tile_bound(P.tokens_q, P.group, 32, P.n_seqs) * P.heads_kv;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  static std::atomic<unsigned long long> done{0};
  const hipError_t configured = allow_lds((const void*)seq_token_kernel<D>, LDS, &done);
  if (configured != hipSuccess) return configured;
  hipLaunchKernelGGL(seq_token_kernel<D>, dim3((unsigned)blocks, (unsigned)P.ranges), dim3(64 * NW), LDS, st, P);
  return hipGetLastError();
}

template <typename E>
hipError_t launch_seq_join(const SeqParams<E>& P, hipStream_t st) {
  const long long rows = (long long)P.tokens_q * P.group;
  auto go = [&](auto dc) -> hipError_t {
    constexpr int D = decltype(dc)::value;
    const bool many = P.ranges >= 8;
    const long long per = many ? 256 / (D / 4) / 4 : 256 / (D / 4), blocks = (rows + per - 1) / per;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks, (unsigned)P.heads_kv);
    if (many) hipLaunchKernelGGL((seq_join_kernel<E, D, 4>), grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL((seq_join_kernel<E, D, 1>), grid, dim3(256), 0, st, P);
    return hipGetLastError();
  };
  const int D = seq_padded(P.d);
  return D == 64 ? go(std::integral_constant<int, 64>{}) : D == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 256>{});
}

template hipError_t launch_seq_token<64>(const SeqParams<bf16_t>&, hipStream_t);
template hipError_t launch_seq_token<128>(const SeqParams<bf16_t>&, hipStream_t);
template hipError_t launch_seq_join<float>(const SeqParams<float>&, hipStream_t);
template hipError_t launch_seq_join<bf16_t>(const SeqParams<bf16_t>&, hipStream_t);

}  // namespace vm
