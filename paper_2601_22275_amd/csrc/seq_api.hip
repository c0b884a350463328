// C entry points of include/vmonarch_sequence.h: validation, workspaces, and which kernel a call takes.
#include <math.h>

#include <cmath>

#include "seq.h"
#include "../../include/vmonarch.h"

using namespace vm;

namespace {

hipStream_t as_stream(void* s) { return (hipStream_t)s; }

int hip_result(hipError_t e, const char* what) {
  return e == hipSuccess ? VMONARCH_OK : api_fail(VMONARCH_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Kernels count tokens, packed rows and keys in 32 bits, and look some tiles (and 64 ranges, each rounded up to 64 keys) past the last
constexpr long long kMostTokens = 0x7fff0000LL;

struct Checked {
  bool aligned = true;  // every row of every tensor seen starts on a 16-byte boundary
};

// A token tensor of `heads` heads and `tokens` tokens; what = its name in an error
int check_tokens(const char* what, const vmonarch_tokens* x, long long tokens, int heads, size_t elem, bool output, Checked* c) {
  if (x == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null %s", what);
  if (tokens > 0 && x->data == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null %s.data", what);
  if (((uintptr_t)x->data % elem) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "%s.data is not aligned to its elements", what);
  if (x->token_stride < 0 || x->head_stride < 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "negative strides of %s", what);
  if (output && ((tokens > 1 && x->token_stride == 0) || (heads > 1 && x->head_stride == 0)))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "%s is written and has a stride of zero", what);
  if (((uintptr_t)x->data | (uintptr_t)(x->token_stride * (long long)elem) | (uintptr_t)(x->head_stride * (long long)elem)) & 15) c->aligned = false;
  return VMONARCH_OK;
}

int check_sizes(int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d) {
  if (n_seqs < 1 || tokens_q < 0 || tokens_k < 0 || heads_q < 1 || heads_kv < 1 || d < 1)
    return api_fail(VMONARCH_ERR_INVALID_ARG, "sizes out of range (n_seqs=%d tokens=%lld, %lld heads=%d, %d d=%d)", n_seqs, tokens_q, tokens_k, heads_q,
                    heads_kv, d);
  if (heads_q % heads_kv != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "heads_q=%d is no multiple of heads_kv=%d", heads_q, heads_kv);
  if (d > 256) return api_fail(VMONARCH_ERR_UNSUPPORTED, "d=%d exceeds 256", d);
  if (heads_q > 65535) return api_fail(VMONARCH_ERR_UNSUPPORTED, "heads_q=%d exceeds 65535", heads_q);
  if (n_seqs > 0x3fffffff) return api_fail(VMONARCH_ERR_UNSUPPORTED, "more than 2^30 - 1 sequences");
  if (tokens_q > kMostTokens || tokens_k > kMostTokens) return api_fail(VMONARCH_ERR_UNSUPPORTED, "more than 2^31 - 65536 tokens");
  if (tokens_q * (heads_q / heads_kv) > kMostTokens) return api_fail(VMONARCH_ERR_UNSUPPORTED, "more rows of queries than one launch takes");
  return VMONARCH_OK;
}

int check_scale(float scale) {
  if (!(scale > 0.f) || std::isinf(scale)) return api_fail(VMONARCH_ERR_INVALID_ARG, "scale must be positive and finite");
  return VMONARCH_OK;
}

int check_starts(const int32_t* starts, const char* what) {
  if (starts == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null %s", what);
  if (((uintptr_t)starts & 3) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "%s is not aligned to its elements", what);
  return VMONARCH_OK;
}

int check_cache(const vmonarch_cache* c, int heads_kv, size_t elem, bool output, Checked* chk) {
  if (c == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null cache");
  if (c->k == nullptr || c->v == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null cache.k or cache.v");
  if (c->n_pages < 1 || c->page_size < 1 || c->table_width < 1)
    return api_fail(VMONARCH_ERR_INVALID_ARG, "sizes must be positive (n_pages=%d page_size=%d table_width=%d)", c->n_pages, c->page_size, c->table_width);
  if (c->table_stride < 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "negative cache.table_stride");
  if ((long long)c->table_width * c->page_size > kMostTokens)
    return api_fail(VMONARCH_ERR_UNSUPPORTED, "a row of the table has room for more than 2^31 - 65536 tokens");
  int rc = check_starts(c->table, "cache.table");
  if (!rc) rc = check_starts(c->lengths, "cache.lengths");
  if (rc) return rc;
  const struct { const char* what; void* p; long long page, t, h; } x[2] = {
      {"cache.k", c->k, c->k_page_stride, c->k_token_stride, c->k_head_stride}, {"cache.v", c->v, c->v_page_stride, c->v_token_stride, c->v_head_stride}};
  for (const auto& a : x) {
    if (((uintptr_t)a.p % elem) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "%s is not aligned to its elements", a.what);
    if (a.page < 0 || a.t < 0 || a.h < 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "negative strides of %s", a.what);
    if (output && ((c->n_pages > 1 && a.page == 0) || (c->page_size > 1 && a.t == 0) || (heads_kv > 1 && a.h == 0)))
      return api_fail(VMONARCH_ERR_INVALID_ARG, "%s is written and has a stride of zero", a.what);
    if (((uintptr_t)a.p | (uintptr_t)(a.page * (long long)elem) | (uintptr_t)(a.t * (long long)elem) | (uintptr_t)(a.h * (long long)elem)) & 15)
      chk->aligned = false;
  }
  return VMONARCH_OK;
}

template <typename E>
Rows<E> rows(const vmonarch_tokens* x) {
  return {(E*)x->data, x->token_stride, x->head_stride};
}
template <typename E>
KeyRows<E> key_rows(const vmonarch_tokens* x) {
  return {(const E*)x->data, x->token_stride, x->head_stride, 0};
}

// ---- rotary ---------------------------------------------------------------------------------------------------------------------
int check_plan(const vmonarch_rotary_plan* p, int d, int* pairs) {
  if (p == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null plan");
  if (p->struct_bytes != sizeof(vmonarch_rotary_plan))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "plan.struct_bytes is %u, this library's vmonarch_rotary_plan has %zu bytes", p->struct_bytes,
                    sizeof(vmonarch_rotary_plan));
  if (p->layout != VMONARCH_ROTARY_HALF && p->layout != VMONARCH_ROTARY_INTERLEAVED) return api_fail(VMONARCH_ERR_INVALID_ARG, "unknown plan.layout %d", p->layout);
  if (p->axes < 1 || p->axes > 3) return api_fail(VMONARCH_ERR_INVALID_ARG, "plan.axes is 1 to 3");
  int n = 0;
  for (int a = 0; a < p->axes; ++a) {
    if (p->axis_pairs[a] < 1 || p->axis_pairs[a] > VMONARCH_ROTARY_MAX_PAIRS) return api_fail(VMONARCH_ERR_INVALID_ARG, "plan.axis_pairs[%d] is %d", a, p->axis_pairs[a]);
    n += p->axis_pairs[a];
  }
  if (n > VMONARCH_ROTARY_MAX_PAIRS) return api_fail(VMONARCH_ERR_INVALID_ARG, "plan has %d pairs, %d at most", n, VMONARCH_ROTARY_MAX_PAIRS);
  if (!std::isfinite(p->amplitude)) return api_fail(VMONARCH_ERR_INVALID_ARG, "plan.amplitude must be finite");
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(p->frequency[i])) return api_fail(VMONARCH_ERR_INVALID_ARG, "plan.frequency[%d] must be finite", i);
  if (d > 0 && 2 * n > d) return api_fail(VMONARCH_ERR_INVALID_ARG, "plan turns %d channels, a head has %d", 2 * n, d);
  *pairs = n;
  return VMONARCH_OK;
}

void plan_params(const vmonarch_rotary_plan* p, int pairs, RotaryParams* P, RotaryTurns* F) {
  constexpr double kTurn = 6.283185307179586476925286766559;
  for (int i = 0; i < pairs; ++i) F->per_position[i] = p->frequency[i] / kTurn;
  P->interleaved = p->layout == VMONARCH_ROTARY_INTERLEAVED;
  P->amplitude = (float)p->amplitude;
  P->axis_end[0] = p->axis_pairs[0];
  P->axis_end[1] = p->axes > 1 ? p->axis_pairs[0] + p->axis_pairs[1] : pairs;
  P->axis_end[2] = pairs;
}

// Whether the pieces of `elem`-byte channels a thread handles can be 16 bytes: a pair's partner lies in the same piece (interleaved) or at the same
// place of another (half, pairs a multiple of a piece)
bool wide_pieces(int interleaved, int pairs, int d, size_t elem) {
  const int v = 16 / (int)elem;
  return d % v == 0 && (interleaved || pairs % v == 0);
}

int rotary_impl(const vmonarch_tokens* q, const vmonarch_tokens* q_out, int heads_q, const vmonarch_tokens* k, const vmonarch_tokens* k_out, int heads_k,
                long long tokens, int d, const int32_t* positions, long long axis_stride, const vmonarch_rotary_plan* plan, int backward, size_t elem,
                void* stream) {
  if (tokens < 0 || heads_q < 1 || heads_k < 0 || d < 1)
    return api_fail(VMONARCH_ERR_INVALID_ARG, "sizes out of range (tokens=%lld heads=%d, %d d=%d)", tokens, heads_q, heads_k, d);
  if (d > 256) return api_fail(VMONARCH_ERR_UNSUPPORTED, "d=%d exceeds 256", d);
  if (heads_q > 65535 || heads_k > 65535) return api_fail(VMONARCH_ERR_UNSUPPORTED, "more than 65535 heads");
  if (tokens > kMostTokens) return api_fail(VMONARCH_ERR_UNSUPPORTED, "more than 2^31 - 65536 tokens");
  if ((k == nullptr) != (heads_k == 0) || (k == nullptr) != (k_out == nullptr))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "k, k_out and heads_k must be given together or not at all");
  int pairs = 0;
  Checked c;
  int rc = check_plan(plan, d, &pairs);
  if (!rc) rc = check_tokens("q", q, tokens, heads_q, elem, false, &c);
  if (!rc) rc = check_tokens("q_out", q_out, tokens, heads_q, elem, true, &c);
  if (!rc && k) rc = check_tokens("k", k, tokens, heads_k, elem, false, &c);
  if (!rc && k) rc = check_tokens("k_out", k_out, tokens, heads_k, elem, true, &c);
  if (!rc && tokens > 0) rc = check_starts(positions, "positions");
  if (rc) return rc;
  const vmonarch_tokens* in[2] = {q, k};
  const vmonarch_tokens* out[2] = {q_out, k_out};
  for (int x = 0; x < (k ? 2 : 1); ++x)
    if (in[x]->data == out[x]->data && (in[x]->token_stride != out[x]->token_stride || in[x]->head_stride != out[x]->head_stride))
      return api_fail(VMONARCH_ERR_INVALID_ARG, "an output in place of its input must have its strides");
  if (k && tokens > 0 && (q_out->data == k_out->data || q_out->data == k->data || k_out->data == q->data))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "q_out and k_out must not be another tensor of the call");
  if (axis_stride < 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "negative axis_stride");
  if (tokens == 0) return VMONARCH_OK;
  RotaryParams P = {};
  RotaryTurns F;
  plan_params(plan, pairs, &P, &F);
  for (int x = 0; x < (k ? 2 : 1); ++x) {
    P.in[x] = in[x]->data; P.in_t[x] = in[x]->token_stride; P.in_h[x] = in[x]->head_stride;
    P.out[x] = out[x]->data; P.out_t[x] = out[x]->token_stride; P.out_h[x] = out[x]->head_stride;
    P.turned[x] = pairs;
  }
  P.heads[0] = heads_q; P.heads[1] = heads_k;
  P.tokens = (int)tokens; P.d = d;
  P.positions = positions; P.axis_stride = axis_stride;
  P.sign = backward ? -1.f : 1.f;
  return hip_result(launch_rotary(P, F, (int)elem, c.aligned && wide_pieces(P.interleaved, pairs, d, elem), as_stream(stream)), "rotary launch");
}

int append_impl(const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_cache* cache, const int32_t* q_starts, int n_seqs, long long tokens,
                int heads_kv, int d, const vmonarch_rotary_plan* plan, const int32_t* positions, long long axis_stride, size_t elem, void* stream) {
  Checked c;
  int pairs = 0;
  int rc = check_sizes(n_seqs, tokens, 0, heads_kv, heads_kv, d);
  if (!rc) rc = check_starts(q_starts, "q_starts");
  if (!rc) rc = check_tokens("k", k, tokens, heads_kv, elem, false, &c);
  if (!rc) rc = check_tokens("v", v, tokens, heads_kv, elem, false, &c);
  if (!rc) rc = check_cache(cache, heads_kv, elem, true, &c);
  if (!rc && plan) rc = check_plan(plan, d, &pairs);
  if (rc) return rc;
  if (plan == nullptr && positions != nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "positions without a plan");
  if (plan != nullptr && positions == nullptr && plan->axes != 1) return api_fail(VMONARCH_ERR_INVALID_ARG, "a plan of %d axes needs positions", plan->axes);
  if (positions != nullptr && (rc = check_starts(positions, "positions")) != 0) return rc;
  if (axis_stride < 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "negative axis_stride");
  if (tokens == 0) return VMONARCH_OK;
  RotaryParams P = {};
  RotaryTurns F;
  P.amplitude = 1.f;
  P.interleaved = 1;
  if (plan) plan_params(plan, pairs, &P, &F);
  P.sign = 1.f;
  P.in[0] = k->data; P.in_t[0] = k->token_stride; P.in_h[0] = k->head_stride;
  P.in[1] = v->data; P.in_t[1] = v->token_stride; P.in_h[1] = v->head_stride;
  P.out[0] = cache->k; P.out_page[0] = cache->k_page_stride; P.out_t[0] = cache->k_token_stride; P.out_h[0] = cache->k_head_stride;
  P.out[1] = cache->v; P.out_page[1] = cache->v_page_stride; P.out_t[1] = cache->v_token_stride; P.out_h[1] = cache->v_head_stride;
  P.turned[0] = pairs;
  P.heads[0] = P.heads[1] = heads_kv;
  P.tokens = (int)tokens; P.d = d;
  P.positions = positions; P.axis_stride = axis_stride;
  P.starts = q_starts; P.n_seqs = n_seqs;
  P.lengths = cache->lengths; P.table = cache->table; P.table_stride = cache->table_stride; P.table_width = cache->table_width;
  P.page_size = cache->page_size; P.n_pages = cache->n_pages;
  return hip_result(launch_rotary(P, F, (int)elem, c.aligned && wide_pieces(P.interleaved, pairs, d, elem), as_stream(stream)), "paged_append launch");
}

// Pages: whether the rows go to the kernel for few of them, and into how many ranges the keys are cut
struct PagedPlan {
  bool few;
  int ranges;
};
PagedPlan paged_plan(long long table_keys, int n_seqs, long long tokens, int heads_kv, int group, bool causal) {
  PagedPlan p;
  const long long rows = tokens * group;
  p.few = rows <= 32LL * n_seqs;
  const long long blocks = tile_bound(tokens, group, p.few ? 32 : 128, n_seqs) * heads_kv;
  const long long shortest = p.few ? 256 : 512, slots = 2LL * compute_units();
  long long r = 1;
  if (p.few) {
    // Small workgroups that stream the cache, eight for every compute unit in turn (16 tokens over up to 16,384 keys: four 145 us, eight 136,
    // sixteen 143).
    r = (4 * slots + blocks - 1) / blocks;
  } else if (slots / blocks >= 3) {
    // Two on a unit at once: as many ranges as one such round holds (chunks of up to 390 tokens over up to 8190, 12 heads, d = 128, 120 workgroups a
    // range, us: 3 102, 4 91, 5 106, 8 107).
    r = slots / blocks;
  } else {
    // Up to five.  The unit of time is an uncut workgroup's.  Sequences of different length wait for the last piece, half of its length is for the
    // balance to spare; the pieces of one sequence are alike and take whole rounds, unless it is short and causal.  A range's partial results cost
    // what 350 keys do (us by ranges: 4 x up to 2048 causal tokens on up to 32,768 keys, 556 workgroups, 1 1272, 2 1129, 4 1066, 5 1071, 8 1109; one
    // sequence: 2912 on 20,000, 276 workgroups, 1 511, 3 424, 4 440, 5 413; 5376 on 10,000, 504, 1 335, 2 358, 5 387; 8192 causal on 32,768, 768, 1
    // 1621, 2 1448, 5 1498; 12,000 causal on themselves, 1128, 1 471, 2 528, 5 623).
    const double each = (double)tokens / n_seqs, load = (double)blocks / slots;
    const double keys = fmax(256.0, (n_seqs == 1 ? 1.0 : 0.5) * table_keys - (causal ? 0.5 * each : 0.0));
    const bool alike = n_seqs == 1 && !(causal && 4 * tokens > table_keys);
    double least = 0;
    for (int x = 1; x <= 5; ++x) {
      const double time = (alike ? (double)((blocks * x + slots - 1) / slots) / x : n_seqs == 1 ? fmax(1.0 / x, load) : load + 1.0 / x) +
                          (x > 1 ? load * 350 * x / keys : 0);
      if (x == 1 || time < least) {
        least = time;
        r = x;
      }
    }
  }
  if (r > (table_keys + shortest - 1) / shortest) r = (table_keys + shortest - 1) / shortest;
  if (r < 1) r = 1;
  p.ranges = r > 64 ? 64 : (int)r;
  return p;
}

template <typename E>
hipError_t launch_attention(const SeqParams<E>& P, bool few, hipStream_t st) {
  hipError_t e;
  if constexpr (sizeof(E) == 2) {
    // (packed keys: 64 rows of an LDS tile lie within 2^31 bytes)
    if (P.aligned && P.d <= 128 && (P.page_size > 0 || (P.k.t < (1 << 24) && P.v.t < (1 << 24)))) {
      if (few) e = P.d <= 64 ? launch_seq_token<64>(P, st) : launch_seq_token<128>(P, st);
      else e = P.d <= 64 ? launch_seq_attention_mfma<64>(P, st) : launch_seq_attention_mfma<128>(P, st);
    } else {
      e = launch_seq_attention_general<E>(P, st);
    }
  } else {
    e = launch_seq_attention_general<E>(P, st);
  }
  return e == hipSuccess && P.ranges > 1 ? launch_seq_join<E>(P, st) : e;
}

// Whether the bf16 matrix units take a backward pass: seq_bwd.hip, else seq_general.hip
template <typename E>
bool bwd_on_bf16_units(bool aligned, int d) {
  return sizeof(E) == 2 && aligned && d <= 128;
}

template <typename E>
hipError_t launch_attention_bwd(const SeqParams<E>& P, hipStream_t st) {
  if constexpr (sizeof(E) == 2) {
    if (bwd_on_bf16_units<E>(P.aligned, P.d)) return P.d <= 64 ? launch_seq_bwd_mfma<64>(P, st) : launch_seq_bwd_mfma<128>(P, st);
  }
  return launch_seq_attention_bwd_general<E>(P, st);
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
template <typename E>
int packed_impl(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_tokens* out, float* lse,
                const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d,
                float scale, int causal, void* stream) {
  Checked c;
  int rc = check_sizes(n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d);
  if (!rc) rc = check_scale(scale);
  if (!rc) rc = check_starts(q_starts, "q_starts");
  if (!rc) rc = check_starts(k_starts, "k_starts");
  if (!rc) rc = check_tokens("q", q, tokens_q, heads_q, sizeof(E), false, &c);
  if (!rc) rc = check_tokens("k", k, tokens_k, heads_kv, sizeof(E), false, &c);
  if (!rc) rc = check_tokens("v", v, tokens_k, heads_kv, sizeof(E), false, &c);
  if (!rc) rc = check_tokens("out", out, tokens_q, heads_q, sizeof(E), true, &c);
  if (rc) return rc;
  if (((uintptr_t)lse & 3) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "lse is not aligned to its elements");
  if (tokens_q == 0) return VMONARCH_OK;
  if (out->data == q->data || out->data == k->data || out->data == v->data) return api_fail(VMONARCH_ERR_INVALID_ARG, "out must not be an input");
  SeqParams<E> P = {};
  P.q = rows<const E>(q); P.k = key_rows<E>(k); P.v = key_rows<E>(v); P.out = rows<E>(out);
  P.lse = lse;
  P.q_starts = q_starts; P.k_starts = k_starts; P.n_seqs = n_seqs;
  P.tokens_q = (int)tokens_q; P.tokens_k = (int)tokens_k;
  P.heads_kv = heads_kv; P.group = heads_q / heads_kv; P.d = d;
  P.causal = causal != 0; P.scale = scale;
  P.aligned = c.aligned && d % (16 / (int)sizeof(E)) == 0;
  return hip_result(launch_attention<E>(P, false, as_stream(stream)), "packed_attention launch");
}

// Workspace of the backward pass: two statistics per query row, then (bf16 matrix units) the partial dK and dV of the ranges of rows
struct BwdLayout {
  size_t parts, total;
  int ranges;
};
BwdLayout bwd_layout(bool bf16_units, int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d) {
  BwdLayout l;
  l.ranges = bf16_units ? seq_bwd_ranges(n_seqs, tokens_q, tokens_k, heads_kv, heads_q / heads_kv) : 1;
  l.parts = ((size_t)tokens_q * heads_q * 2 * sizeof(float) + 255) & ~(size_t)255;
  l.total = l.parts;
  if (l.ranges > 1) l.total += ((size_t)l.ranges * 2 * tokens_k * heads_kv * seq_padded(d) * sizeof(float) + 255) & ~(size_t)255;
  return l;
}

// (rows taken to be aligned: less is needed where they are not)
template <typename E>
size_t bwd_workspace(int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d) {
  if (n_seqs < 1 || tokens_q < 1 || tokens_k < 0 || heads_kv < 1 || heads_q < heads_kv || heads_q % heads_kv != 0 || d < 1 || d > 256) return 0;
  return bwd_layout(bwd_on_bf16_units<E>(d % (16 / (int)sizeof(E)) == 0, d), n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d).total;
}

template <typename E>
int packed_bwd_impl(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_tokens* out, const vmonarch_tokens* d_out,
                    const float* lse, const vmonarch_tokens* dq, const vmonarch_tokens* dk, const vmonarch_tokens* dv, const int32_t* q_starts,
                    const int32_t* k_starts, int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d, float scale,
                    int causal, void* workspace, size_t workspace_bytes, void* stream) {
  Checked c;
  int rc = check_sizes(n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d);
  if (!rc) rc = check_scale(scale);
  if (!rc) rc = check_starts(q_starts, "q_starts");
  if (!rc) rc = check_starts(k_starts, "k_starts");
  const struct { const char* what; const vmonarch_tokens* x; bool keys, output; } all[] = {
      {"q", q, false, false}, {"k", k, true, false}, {"v", v, true, false}, {"out", out, false, false}, {"d_out", d_out, false, false},
      {"dq", dq, false, true}, {"dk", dk, true, true}, {"dv", dv, true, true}};
  for (const auto& a : all)
    if (!rc) rc = check_tokens(a.what, a.x, a.keys ? tokens_k : tokens_q, a.keys ? heads_kv : heads_q, sizeof(E), a.output, &c);
  if (rc) return rc;
  for (const auto& a : all)
    for (const auto& b : all)
      if (a.output && &a != &b && a.x->data == b.x->data && a.x->data != nullptr)
        return api_fail(VMONARCH_ERR_INVALID_ARG, "%s must not be %s", a.what, b.what);
  if (dq == dk || dq == dv || dk == dv) return api_fail(VMONARCH_ERR_INVALID_ARG, "dq, dk and dv must differ");
  if (tokens_q > 0 && lse == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null lse");
  if (((uintptr_t)lse & 3) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "lse is not aligned to its elements");
  if (((uintptr_t)workspace & 255) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if ((workspace == nullptr) != (workspace_bytes == 0))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "workspace and workspace_bytes must both be zero or both non-zero");
  if (tokens_q == 0 && tokens_k == 0) return VMONARCH_OK;
  SeqParams<E> P = {};
  P.aligned = c.aligned && d % (16 / (int)sizeof(E)) == 0;
  P.ranges = 1;
  if (tokens_q > 0) {
    const BwdLayout l = bwd_layout(bwd_on_bf16_units<E>(P.aligned, d), n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d);
    char* ws = (char*)api_workspace(l.total, &rc, workspace, workspace_bytes, as_stream(stream));
    if (rc) return rc;
    P.delta = (float*)ws;
    P.part_o = (float*)(ws + l.parts);
    P.ranges = l.ranges;
  }
  P.q = rows<const E>(q); P.k = key_rows<E>(k); P.v = key_rows<E>(v); P.o = rows<const E>(out); P.d_out = rows<const E>(d_out);
  P.dq = rows<E>(dq); P.dk = rows<E>(dk); P.dv = rows<E>(dv);
  P.lse = const_cast<float*>(lse);
  P.q_starts = q_starts; P.k_starts = k_starts; P.n_seqs = n_seqs;
  P.tokens_q = (int)tokens_q; P.tokens_k = (int)tokens_k;
  P.heads_kv = heads_kv; P.group = heads_q / heads_kv; P.d = d;
  P.causal = causal != 0; P.scale = scale;
  return hip_result(launch_attention_bwd<E>(P, as_stream(stream)), "packed_attention_bwd launch");
}

template <typename E>
int paged_impl(const vmonarch_tokens* q, const vmonarch_cache* cache, const vmonarch_tokens* out, const int32_t* q_starts, int n_seqs,
               long long tokens, int heads_q, int heads_kv, int d, float scale, int causal, void* workspace, size_t workspace_bytes, void* stream) {
  Checked c;
  int rc = check_sizes(n_seqs, tokens, 0, heads_q, heads_kv, d);
  if (!rc) rc = check_scale(scale);
  if (!rc) rc = check_starts(q_starts, "q_starts");
  if (!rc) rc = check_tokens("q", q, tokens, heads_q, sizeof(E), false, &c);
  if (!rc) rc = check_tokens("out", out, tokens, heads_q, sizeof(E), true, &c);
  if (!rc) rc = check_cache(cache, heads_kv, sizeof(E), false, &c);
  if (rc) return rc;
  if (((uintptr_t)workspace & 255) != 0) return api_fail(VMONARCH_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if ((workspace == nullptr) != (workspace_bytes == 0))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "workspace and workspace_bytes must both be zero or both non-zero");
  if (tokens == 0) return VMONARCH_OK;
  if (out->data == q->data || out->data == cache->k || out->data == cache->v) return api_fail(VMONARCH_ERR_INVALID_ARG, "out must not be an input");
  SeqParams<E> P = {};
  P.q = rows<const E>(q); P.out = rows<E>(out);
  P.k = {(const E*)cache->k, cache->k_token_stride, cache->k_head_stride, cache->k_page_stride};
  P.v = {(const E*)cache->v, cache->v_token_stride, cache->v_head_stride, cache->v_page_stride};
  P.q_starts = q_starts; P.n_seqs = n_seqs;
  P.lengths = cache->lengths; P.table = cache->table; P.table_stride = cache->table_stride; P.table_width = cache->table_width;
  P.page_size = cache->page_size; P.n_pages = cache->n_pages;
  P.tokens_q = (int)tokens;
  P.heads_kv = heads_kv; P.group = heads_q / heads_kv; P.d = d;
  P.causal = causal != 0; P.scale = scale;
  P.aligned = c.aligned && d % (16 / (int)sizeof(E)) == 0;
  const PagedPlan plan = paged_plan((long long)cache->table_width * cache->page_size, n_seqs, tokens, heads_kv, P.group, causal != 0);
  P.ranges = plan.ranges;
  if (plan.ranges > 1) {
    const size_t need = vmonarch_paged_attention_workspace_bytes(cache, n_seqs, tokens, heads_q, heads_kv, d);
    P.part_o = (float*)api_workspace(need, &rc, workspace, workspace_bytes, as_stream(stream));
    if (rc) return rc;
    P.part_s = P.part_o + (size_t)plan.ranges * tokens * heads_q * seq_padded(d);
  }
  return hip_result(launch_attention<E>(P, plan.few, as_stream(stream)), "paged_attention launch");
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

int vmonarch_rotary_init(vmonarch_rotary_plan* plan, int layout, double base, int axes, const int* axis_pairs_host) {
  if (plan == nullptr || axis_pairs_host == nullptr) return api_fail(VMONARCH_ERR_INVALID_ARG, "null plan or axis_pairs");
  if (!(base > 0.0) || std::isinf(base)) return api_fail(VMONARCH_ERR_INVALID_ARG, "base must be positive and finite");
  if (axes < 1 || axes > 3) return api_fail(VMONARCH_ERR_INVALID_ARG, "axes is 1 to 3");
  vmonarch_rotary_plan p = {};
  p.struct_bytes = (uint32_t)sizeof(p);
  p.layout = layout;
  p.axes = axes;
  p.amplitude = 1.0;
  for (int a = 0; a < axes; ++a) p.axis_pairs[a] = axis_pairs_host[a];
  int pairs = 0;
  const int rc = check_plan(&p, 0, &pairs);
  if (rc) return rc;
  for (int a = 0, n = 0; a < axes; ++a)
    for (int i = 0; i < p.axis_pairs[a]; ++i) p.frequency[n++] = pow(base, -(double)i / p.axis_pairs[a]);
  *plan = p;
  return VMONARCH_OK;
}

int vmonarch_rotary_scale(vmonarch_rotary_plan* plan, double factor, double context, double low_turns, double high_turns) {
  int pairs = 0;
  const int rc = check_plan(plan, 0, &pairs);
  if (rc) return rc;
  if (!(factor > 0.0) || std::isinf(factor)) return api_fail(VMONARCH_ERR_INVALID_ARG, "factor must be positive and finite");
  if (!(context >= 0.0) || std::isinf(context)) return api_fail(VMONARCH_ERR_INVALID_ARG, "context must be finite and not negative");
  if (context > 0.0 && (!(low_turns < high_turns) || std::isinf(low_turns) || std::isinf(high_turns)))
    return api_fail(VMONARCH_ERR_INVALID_ARG, "low_turns must be less than high_turns, both finite");
  constexpr double kTurn = 6.283185307179586476925286766559;
  for (int i = 0; i < pairs; ++i) {
    double keep = 0.0;
    if (context > 0.0) keep = fmin(fmax((context * plan->frequency[i] / kTurn - low_turns) / (high_turns - low_turns), 0.0), 1.0);
    plan->frequency[i] *= keep + (1.0 - keep) / factor;
  }
  return VMONARCH_OK;
}

int vmonarch_rotary(const vmonarch_tokens* q, const vmonarch_tokens* q_out, int heads_q, const vmonarch_tokens* k, const vmonarch_tokens* k_out,
                    int heads_k, long long tokens, int d, const int32_t* positions, long long axis_stride, const vmonarch_rotary_plan* plan,
                    int backward, void* stream) {
  return rotary_impl(q, q_out, heads_q, k, k_out, heads_k, tokens, d, positions, axis_stride, plan, backward, 2, stream);
}
int vmonarch_rotary_f32(const vmonarch_tokens* q, const vmonarch_tokens* q_out, int heads_q, const vmonarch_tokens* k, const vmonarch_tokens* k_out,
                        int heads_k, long long tokens, int d, const int32_t* positions, long long axis_stride, const vmonarch_rotary_plan* plan,
                        int backward, void* stream) {
  return rotary_impl(q, q_out, heads_q, k, k_out, heads_k, tokens, d, positions, axis_stride, plan, backward, 4, stream);
}

int vmonarch_packed_attention(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_tokens* out, float* lse,
                              const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q, long long tokens_k, int heads_q,
                              int heads_kv, int d, float scale, int causal, void* stream) {
  return packed_impl<bf16_t>(q, k, v, out, lse, q_starts, k_starts, n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d, scale, causal, stream);
}
int vmonarch_packed_attention_f32(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_tokens* out, float* lse,
                                  const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q, long long tokens_k, int heads_q,
                                  int heads_kv, int d, float scale, int causal, void* stream) {
  return packed_impl<float>(q, k, v, out, lse, q_starts, k_starts, n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d, scale, causal, stream);
}

size_t vmonarch_packed_attention_bwd_workspace_bytes(int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d) {
  return bwd_workspace<bf16_t>(n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d);
}
size_t vmonarch_packed_attention_bwd_workspace_bytes_f32(int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d) {
  return bwd_workspace<float>(n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d);
}
int vmonarch_packed_attention_bwd(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_tokens* out,
                                  const vmonarch_tokens* d_out, const float* lse, const vmonarch_tokens* dq, const vmonarch_tokens* dk,
                                  const vmonarch_tokens* dv, const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q,
                                  long long tokens_k, int heads_q, int heads_kv, int d, float scale, int causal, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  return packed_bwd_impl<bf16_t>(q, k, v, out, d_out, lse, dq, dk, dv, q_starts, k_starts, n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d, scale,
                                 causal, workspace, workspace_bytes, stream);
}
int vmonarch_packed_attention_bwd_f32(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_tokens* out,
                                      const vmonarch_tokens* d_out, const float* lse, const vmonarch_tokens* dq, const vmonarch_tokens* dk,
                                      const vmonarch_tokens* dv, const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q,
                                      long long tokens_k, int heads_q, int heads_kv, int d, float scale, int causal, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  return packed_bwd_impl<float>(q, k, v, out, d_out, lse, dq, dk, dv, q_starts, k_starts, n_seqs, tokens_q, tokens_k, heads_q, heads_kv, d, scale,
                                causal, workspace, workspace_bytes, stream);
}

int vmonarch_paged_append(const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_cache* cache, const int32_t* q_starts, int n_seqs,
                          long long tokens, int heads_kv, int d, const vmonarch_rotary_plan* plan, const int32_t* positions, long long axis_stride,
                          void* stream) {
  return append_impl(k, v, cache, q_starts, n_seqs, tokens, heads_kv, d, plan, positions, axis_stride, 2, stream);
}
int vmonarch_paged_append_f32(const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_cache* cache, const int32_t* q_starts, int n_seqs,
                              long long tokens, int heads_kv, int d, const vmonarch_rotary_plan* plan, const int32_t* positions,
                              long long axis_stride, void* stream) {
  return append_impl(k, v, cache, q_starts, n_seqs, tokens, heads_kv, d, plan, positions, axis_stride, 4, stream);
}

size_t vmonarch_paged_attention_workspace_bytes(const vmonarch_cache* cache, int n_seqs, long long tokens, int heads_q, int heads_kv, int d) {
  if (cache == nullptr || cache->table_width < 1 || cache->page_size < 1 || n_seqs < 1 || tokens < 1 || heads_kv < 1 || heads_q < heads_kv ||
      heads_q % heads_kv != 0 || d < 1 || d > 256)
    return 0;
  int ranges = 1;  // with a causal mask or without
  for (const bool causal : {false, true}) {
    const int r = paged_plan((long long)cache->table_width * cache->page_size, n_seqs, tokens, heads_kv, heads_q / heads_kv, causal).ranges;
    if (r > ranges) ranges = r;
  }
  if (ranges < 2) return 0;
  return ((size_t)ranges * tokens * heads_q * (seq_padded(d) + 1) * sizeof(float) + 255) & ~(size_t)255;
}
int vmonarch_paged_attention(const vmonarch_tokens* q, const vmonarch_cache* cache, const vmonarch_tokens* out, const int32_t* q_starts, int n_seqs,
                             long long tokens, int heads_q, int heads_kv, int d, float scale, int causal, void* workspace, size_t workspace_bytes,
                             void* stream) {
  return paged_impl<bf16_t>(q, cache, out, q_starts, n_seqs, tokens, heads_q, heads_kv, d, scale, causal, workspace, workspace_bytes, stream);
}
int vmonarch_paged_attention_f32(const vmonarch_tokens* q, const vmonarch_cache* cache, const vmonarch_tokens* out, const int32_t* q_starts, int n_seqs,
                                 long long tokens, int heads_q, int heads_kv, int d, float scale, int causal, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  return paged_impl<float>(q, cache, out, q_starts, n_seqs, tokens, heads_q, heads_kv, d, scale, causal, workspace, workspace_bytes, stream);
}

#pragma GCC visibility pop
}  // extern "C"
