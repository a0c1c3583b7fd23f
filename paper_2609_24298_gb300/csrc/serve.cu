// libcobra device entry points for serving with drafted tokens: norms with the rotation, runs of new
// tokens into the cache, attention of a tree of drafted tokens.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/cobra.h"
#include "append_run.cuh"
#include "launch.cuh"
#include "norm_rope.cuh"
#include "tree.cuh"

using namespace cobra;

namespace {
constexpr int kRopeMaxPos = 1 << 22;
int coarse_rows(int max_pos) { return (max_pos + kRopeFine - 1) / kRopeFine; }
}  // namespace

namespace cobra {
cobra_status take_serve_status(unsigned int* bits) {
  if (cudaMemcpyFromSymbol(bits, g_status, sizeof(*bits)) != cudaSuccess) return COBRA_ECUDA;
  if (*bits) {
    const unsigned int zero = 0;
    if (cudaMemcpyToSymbol(g_status, &zero, sizeof(zero)) != cudaSuccess) return COBRA_ECUDA;
  }
  return COBRA_OK;
}
}  // namespace cobra

// ---------------------------------------------------------------------------------------
// Norms with the rotation
// ---------------------------------------------------------------------------------------
extern "C" cobra_status cobra_norm_rope(const cobra_norm_rope_desc* d, const void* q, const void* k,
                                        const float* q_weight, const float* k_weight, const int* pos,
                                        const float* rope_table, int max_pos, void* q_out, void* k_out, void* stream) {
  if (!d || d->n_tok < 0 || d->n_q_heads < 0 || d->n_k_heads < 0 || d->n_q_heads + (long long)d->n_k_heads < 1 ||
      d->n_q_heads > 65536 || d->n_k_heads > 65536)
    return COBRA_EINVAL;
  if (!d->norm && !rope_table) return COBRA_EINVAL;  // nothing to do
  if (d->norm && !(d->eps >= 0.f && d->eps < INFINITY)) return COBRA_EINVAL;
  if (d->n_tok == 0) return COBRA_OK;  // (empty tensors have no address)
  if ((d->n_q_heads && (!q || !q_out)) || (d->n_k_heads && (!k || !k_out))) return COBRA_EINVAL;
  if (rope_table && (!pos || max_pos < 1 || max_pos > kRopeMaxPos)) return COBRA_EINVAL;
  if (!d->norm && (q_weight || k_weight)) return COBRA_EINVAL;
  if ((rope_table && !aligned(rope_table, 16)) || (pos && !aligned(pos, 4)) || (q_weight && !aligned(q_weight, 16)) ||
      (k_weight && !aligned(k_weight, 16)))
    return COBRA_EALIGN;
  auto side = [](const void* x, void* o, const float* w, long long st, long long sh, long long ot, long long oh, int heads) {
    return NormSide{static_cast<const __nv_bfloat16*>(x), static_cast<__nv_bfloat16*>(o), w, st, sh, ot, oh, heads};
  };
  NormArgs a{};
  a.q = side(q, q_out, q_weight, d->q_stride_tok, d->q_stride_head, d->qo_stride_tok, d->qo_stride_head, d->n_q_heads);
  a.k = side(k, k_out, k_weight, d->k_stride_tok, d->k_stride_head, d->ko_stride_tok, d->ko_stride_head, d->n_k_heads);
  for (const NormSide* s : {&a.q, &a.k})
    if (s->heads && (!aligned(s->x, 16) || !aligned(s->out, 16) || ((s->st | s->sh | s->ot | s->oh) & 7))) return COBRA_EALIGN;
  a.pos = pos;
  a.table = rope_table;
  a.n_coarse = rope_table ? coarse_rows(max_pos) : 0;
  a.n_tok = d->n_tok;
  a.norm = d->norm != 0;
  a.eps = d->eps;
  a.q_groups = (d->n_q_heads + 3) / 4;
  a.groups = a.q_groups + (d->n_k_heads + 3) / 4;
  // groups of four heads per warp: one while the call does not fill the GPU, more (fewer compositions of a
  // token's angles) where every SM has its 64 warps all the same
  const long long units = (long long)d->n_tok * a.groups, room = 64LL * sm_count();
  a.per_warp = (int)std::max(1LL, std::min<long long>(a.groups, units / room));
  const long long warps = (long long)d->n_tok * ((a.groups + a.per_warp - 1) / a.per_warp);
  const long long grid = (warps + kNormThreads / 32 - 1) / (kNormThreads / 32);
  if (grid > 0x7fffffffLL) return COBRA_EINVAL;
  if (launch_pdl(norm_rope_kernel, (unsigned)grid, kNormThreads, 0, (cudaStream_t)stream, a) != cudaSuccess)
    return COBRA_ECUDA;
  return launch_status();
}

// ---------------------------------------------------------------------------------------
// Runs of new tokens
// ---------------------------------------------------------------------------------------
extern "C" cobra_status cobra_rope_table64_bytes(int max_pos, size_t* bytes) {
  if (!bytes || max_pos < 1 || max_pos > kRopeMaxPos) return COBRA_EINVAL;
  *bytes = (size_t)(kRopeFine + coarse_rows(max_pos)) * kD * sizeof(double);
  return COBRA_OK;
}

extern "C" cobra_status cobra_rope_table64(double theta, int max_pos, double* table, size_t table_bytes, void* stream) {
  size_t need = 0;
  const cobra_status st = cobra_rope_table64_bytes(max_pos, &need);
  if (st != COBRA_OK) return st;
  if (!table || !(theta > 0.0) || !(theta < 1e300)) return COBRA_EINVAL;
  if (!aligned(table, 16)) return COBRA_EALIGN;
  if (table_bytes < need) return COBRA_ESPACE;
  const int n_rows = kRopeFine + coarse_rows(max_pos), n = n_rows * (kD / 2);
  if (launch_pdl(rope_table64_kernel, (unsigned)((n + 255) / 256), 256, 0, (cudaStream_t)stream, table, n_rows, theta) !=
      cudaSuccess)
    return COBRA_ECUDA;
  return launch_status();
}

namespace {
template <class C>
cobra_status launch_run(const RunArgs& a, long long units, void* stream) {
  static Granted granted;
  const size_t smem = sizeof(RunSmem<C>) + 1024;
  if (ensure_smem(append_run_kernel<C>, smem, granted) != COBRA_OK) return COBRA_ECUDA;
  const unsigned grid = (unsigned)std::min(units, (long long)C::kPerSm * sm_count());
  if (launch_pdl(append_run_kernel<C>, grid, C::kThreads, smem, (cudaStream_t)stream, a) != cudaSuccess) return COBRA_ECUDA;
  return launch_status();
}
}  // namespace

extern "C" cobra_status cobra_append_tokens(const void* params, const cobra_append_desc* d, const void* k, const void* v,
                                            const int* pos, const int* n_new, const int* index, const double* rope_table,
                                            int max_pos, uint8_t* cache, const int* page_table, void* stream) {
  if (!d || !params || !k || !v || !pos || !cache) return COBRA_EINVAL;
  if (d->k_head0 < 0 || d->v_head0 < 0 || d->n_layers < 1 || d->n_kv_heads < 1 || d->layer_stride < d->n_kv_heads ||
      d->n_seqs < 1 || d->max_new < 0 || d->n_src < 1 || d->rows_per_seq < 0 || d->pages_per_seq < 0)
    return COBRA_EINVAL;
  if (!index && d->n_src < d->max_new) return COBRA_EINVAL;
  if (page_table ? d->pages_per_seq < 1 : d->rows_per_seq < 1) return COBRA_EINVAL;
  if (rope_table && (max_pos < 1 || max_pos > kRopeMaxPos)) return COBRA_EINVAL;
  const long long heads = (long long)d->n_layers * d->n_kv_heads;
  const long long top = std::max(d->k_head0, d->v_head0) + (d->n_layers - 1LL) * d->layer_stride + d->n_kv_heads;
  if (heads > (1 << 24) || top > 0x7fffffffLL) return COBRA_EINVAL;
  const long long rows = d->n_seqs * (((long long)d->max_new + 126) / 128 + 1);  // at most
  if (rows > 0x7fffffffLL) return COBRA_EINVAL;
  if (!aligned(params, 256) || !aligned(cache, 256) || !aligned(k, 2) || !aligned(v, 2) || !aligned(pos, 4) ||
      (n_new && !aligned(n_new, 4)) || (index && !aligned(index, 4)) || (page_table && !aligned(page_table, 4)) ||
      (rope_table && !aligned(rope_table, 16)))
    return COBRA_EALIGN;
  if (d->max_new == 0) return COBRA_OK;
  RunArgs a{};
  a.block = static_cast<const unsigned char*>(params);
  a.x[0] = static_cast<const __nv_bfloat16*>(k);
  a.x[1] = static_cast<const __nv_bfloat16*>(v);
  a.cache = cache;
  a.page_table = page_table;
  a.pos = pos;
  a.n_new = n_new;
  a.index = index;
  a.table = rope_table;
  a.n_coarse = rope_table ? coarse_rows(max_pos) : 0;
  a.sl = d->x_stride_layer;
  a.ss = d->x_stride_seq;
  a.st = d->x_stride_tok;
  a.sh = d->x_stride_head;
  a.head0[0] = d->k_head0;
  a.head0[1] = d->v_head0;
  a.layer_stride = d->layer_stride;
  a.n_layers = d->n_layers;
  a.n_kv = d->n_kv_heads;
  a.n_seqs = d->n_seqs;
  a.max_new = d->max_new;
  a.n_src = d->n_src;
  a.rows_per_seq = d->rows_per_seq;
  a.pages_per_seq = d->pages_per_seq;
  // A row's tokens have to fit a batch.  Below that, small batches where a CTA has one of them or rows have a token
  // or two (a batch holds 32 rows at most).  us, few and mid: a layer of 8 heads, 64 sequences x 7 tokens 15.8 and
  // 17.7, x 10 tokens 23.4 and 20.9; 32 layers, 64 sequences x 1 token 98 and 127, x 2 tokens 132 and 140, 16
  // sequences x 8 tokens 111 and 103.  Mid and many: 32 layers, 64 sequences x 4 tokens 127 and 157.
  const long long tokens = 2 * heads * d->n_seqs * d->max_new, units = 2 * heads * rows;
  if (d->max_new <= 2 || (d->max_new <= RunFew::kTokens && tokens <= (long long)RunFew::kTokens * RunFew::kPerSm * sm_count()))
    return launch_run<RunFew>(a, units, stream);
  return d->max_new <= RunMid::kTokens ? launch_run<RunMid>(a, units, stream) : launch_run<RunMany>(a, units, stream);
}

// ---------------------------------------------------------------------------------------
// Tree attention
// ---------------------------------------------------------------------------------------
namespace {

cobra_status check_tree_desc(const cobra_tree_desc* d) {
  if (!d) return COBRA_EINVAL;
  if (d->k_head0 < 0 || d->v_head0 < 0 || d->n_layers < 1 || d->n_kv_heads < 1 || d->layer_stride < d->n_kv_heads ||
      d->n_seqs < 1 || d->group < 1 || d->group > 16 || d->max_draft < 1 || d->max_draft > kTreeMaxDraft ||
      d->rows_per_seq < 0 || d->pages_per_seq < 0 || d->window < 0 || !(d->softcap >= 0.f) || !(d->softcap < 1e30f))
    return COBRA_EINVAL;
  const long long heads = (long long)d->n_layers * d->n_kv_heads;
  const long long top = std::max(d->k_head0, d->v_head0) + (d->n_layers - 1LL) * d->layer_stride + d->n_kv_heads;
  // cached tokens are counted in ints; the launches' grids are 32 bits wide
  if (top > 0x7fffffffLL || 256LL * d->pages_per_seq > 0x7fffffffLL || 128LL * d->rows_per_seq > 0x7fffffffLL ||
      heads > (1 << 24) || heads * d->n_seqs > (1 << 24))
    return COBRA_EINVAL;
  return COBRA_OK;
}

// Column tiles and the workspace: the layout's pointers are offsets from `base`.
size_t tree_layout_host(const cobra_tree_desc* d, unsigned char* base, TreeArgs& a) {
  const long long heads = (long long)d->n_layers * d->n_kv_heads, cols = (long long)d->max_draft * d->group;
  a.nc = cols <= 16 ? 16 : cols <= 32 ? 32 : 64;
  a.tiles = (int)((cols + a.nc - 1) / a.nc);
  a.chunks = a.nc < kTreeChunk ? 1 : a.tiles * (a.nc / kTreeChunk);
  a.ctas = std::min(sm_count(), kTreeParts);  // (the combine holds a unit's parts at once)
  const size_t S = d->n_seqs, units = (size_t)(heads * d->n_seqs) * a.tiles;
  size_t off = 0;
  auto take = [&](auto*& p, size_t n) {
    using T = std::remove_reference_t<decltype(*p)>;
    p = reinterpret_cast<T*>(base + off);
    off = (off + n * sizeof(T) + 255) / 256 * 256;
  };
  take(a.row0, S);
  take(a.rows, S);
  take(a.live, S);
  take(a.row_bytes, 2);
  take(a.start, 2LL * a.ctas);
  take(a.rpre, S + 1);
  take(a.wpre, (size_t)heads + 1);
  take(a.img, units * 2 * a.nc * 128);
  take(a.col, units * a.nc);
  take(a.draft, (size_t)(heads * d->n_seqs) * cols * kTreePart);
  take(a.part, (units + a.ctas) * a.nc * kTreePart);
  return off;
}

template <int NC, int NCW, bool LARGE>
cobra_status launch_tree_scan_kind(const TreeArgs& a, cudaStream_t s) {
  using Smem = TreeScanSmem<NC, NCW>;
  static Granted granted;
  if (ensure_smem(tree_scan_kernel<NC, NCW, LARGE>, sizeof(Smem) + 1024, granted) != COBRA_OK) return COBRA_ECUDA;
  return launch_pdl(tree_scan_kernel<NC, NCW, LARGE>, (unsigned)a.ctas, Smem::kThreads, sizeof(Smem) + 1024, s, a) == cudaSuccess
             ? COBRA_OK
             : COBRA_ECUDA;
}
template <int NC, int NCW>
cobra_status launch_tree_scan(const TreeArgs& a, cudaStream_t s) {
  return a.cap2 > kTreeCapPlain ? launch_tree_scan_kind<NC, NCW, true>(a, s) : launch_tree_scan_kind<NC, NCW, false>(a, s);
}

}  // namespace

extern "C" cobra_status cobra_tree_workspace_size(const cobra_tree_desc* desc, size_t* bytes) {
  const cobra_status st = check_tree_desc(desc);
  if (st != COBRA_OK) return st;
  if (!bytes) return COBRA_EINVAL;
  TreeArgs a{};
  *bytes = tree_layout_host(desc, nullptr, a);
  return COBRA_OK;
}

extern "C" cobra_status cobra_tree_attn(const void* params, const cobra_tree_desc* d, const void* q, const void* k_draft,
                                        const void* v_draft, const int* n_draft, const uint64_t* tree_mask,
                                        const int* q_pos, const float* slopes, const uint8_t* cache, const int* seq_lens,
                                        const int* page_table, void* out, void* workspace, size_t ws_bytes, void* stream) {
  const cobra_status st = check_tree_desc(d);
  if (st != COBRA_OK) return st;
  if (!params || !q || !cache || !seq_lens || !out || !workspace || !k_draft != !v_draft) return COBRA_EINVAL;
  if (page_table ? d->pages_per_seq < 1 : d->rows_per_seq < 1) return COBRA_EINVAL;
  if (!aligned(params, 256) || !aligned(cache, 256) || !aligned(workspace, 256) || !aligned(q, 2) || !aligned(out, 2) ||
      !aligned(k_draft, 2) || !aligned(v_draft, 2) || !aligned(n_draft, 4) || !aligned(tree_mask, 8) ||
      !aligned(q_pos, 4) || !aligned(slopes, 4) || !aligned(seq_lens, 4) || !aligned(page_table, 4))
    return COBRA_EALIGN;
  TreeArgs a{};
  if (ws_bytes < tree_layout_host(d, static_cast<unsigned char*>(workspace), a)) return COBRA_ESPACE;
  a.block = static_cast<const unsigned char*>(params);
  a.cache = cache;
  a.page_table = page_table;
  a.seq_lens = seq_lens;
  a.n_draft = n_draft;
  a.q_pos = q_pos;
  a.mask = reinterpret_cast<const unsigned long long*>(tree_mask);
  a.slopes = slopes;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.kd = static_cast<const __nv_bfloat16*>(k_draft);
  a.vd = static_cast<const __nv_bfloat16*>(v_draft);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.q_sl = d->q_stride_layer, a.q_ss = d->q_stride_seq, a.q_st = d->q_stride_tok;
  a.d_sl = d->d_stride_layer, a.d_ss = d->d_stride_seq, a.d_st = d->d_stride_tok, a.d_sh = d->d_stride_head;
  a.o_sl = d->o_stride_layer, a.o_ss = d->o_stride_seq, a.o_st = d->o_stride_tok;
  a.k_head0 = d->k_head0, a.v_head0 = d->v_head0, a.layer_stride = d->layer_stride;
  a.n_layers = d->n_layers, a.n_kv = d->n_kv_heads, a.group = d->group, a.n_seqs = d->n_seqs;
  a.max_draft = d->max_draft;
  a.rows_per_seq = d->rows_per_seq, a.pages_per_seq = d->pages_per_seq;
  a.window = d->window;
  a.cap2 = d->softcap * kLog2e;
  a.top_f16 = kTopF16;
  a.top_bf16 = kTopBf16;
  const long long units = (long long)d->n_layers * d->n_kv_heads * d->n_seqs;
  const long long prep = 1 + units * a.chunks * (a.kd ? 2 : 1);
  const long long comb = units * ((d->max_draft * d->group + kTreeCombine - 1) / kTreeCombine);
  cudaStream_t s = (cudaStream_t)stream;
  static Granted prep_granted;
  const size_t prep_smem = std::max(sizeof(TreeProjSmem), sizeof(TreeDraftSmem)) + 1024;
  if (ensure_smem(tree_prepare_kernel, prep_smem, prep_granted) != COBRA_OK) return COBRA_ECUDA;
  if (launch_pdl(tree_prepare_kernel, (unsigned)prep, 256, prep_smem, s, a) != cudaSuccess) return COBRA_ECUDA;
  const long long cols = (long long)d->max_draft * d->group;
  cobra_status r;
  if (cols <= 8)
    r = launch_tree_scan<16, 8>(a, s);
  else if (a.nc == 16)
    r = launch_tree_scan<16, 16>(a, s);
  else if (a.nc == 32)
    r = launch_tree_scan<32, 32>(a, s);
  else
    r = launch_tree_scan<64, 32>(a, s);
  if (r != COBRA_OK) return r;
  if (launch_pdl(tree_combine_kernel, (unsigned)comb, 256, 0, s, a) != cudaSuccess) return COBRA_ECUDA;
  return launch_status();
}
