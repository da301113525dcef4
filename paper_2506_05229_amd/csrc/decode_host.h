// Host side of the decoding operators (included at the end of armt_api.hip): argument checks and launches.
#pragma once

namespace {

constexpr int kMaxSeqs = 65536;

// Head layout of a configuration for the cache; of the fp32 head sizes, those with whole 16-byte rows.
armt_status check_cache(const armt_config* cfg, const armt_kv_cache* cache, int32_t n_rows, Dims* D, KvView* v) {
  ARMT_TRY(check_config(cfg, D));
  if (!cache) return ARMT_ERR_NULL;
  if (!cache->k || !cache->v || !cache->pages || !cache->lens || !cache->row_start) return ARMT_ERR_NULL;
  if (cache->n_seqs < 1 || cache->n_pages < 1 || cache->max_pages < 1 || n_rows < 1) return ARMT_ERR_SHAPE;
  if (cache->page_len < 1 || cache->n_seqs > kMaxSeqs) return ARMT_ERR_SHAPE;
  if (D->dh % 4 || D->dh > 128) return ARMT_ERR_UNSUPPORTED;
  if (cache->page_len < 16 || cache->page_len > 4096 || (cache->page_len & (cache->page_len - 1))) return ARMT_ERR_UNSUPPORTED;
  const int64_t page = (int64_t)D->Hkv * cache->page_len * D->dh, stride = cache->page_stride ? cache->page_stride : page;
  if (stride < page) return ARMT_ERR_SHAPE;
  if (stride * (int64_t)D->esz % 16 || (uintptr_t)cache->k % 16 || (uintptr_t)cache->v % 16) return ARMT_ERR_UNSUPPORTED;
  int shift = 0;
  while ((1 << shift) < cache->page_len) ++shift;
  *v = KvView{cache->pages, cache->lens, cache->row_start, cache->n_seqs, cache->n_pages, cache->max_pages, shift, n_rows, stride};
  return ARMT_OK;
}

// Grid and workspace limits of the attention; false: too large for a launch.
bool attention_plan(const Dims& D, int32_t n_seqs, int32_t max_pages, int32_t page_len, int32_t n_rows, int32_t max_rows, KvPlan* p) {
  if ((int64_t)max_rows * (D.H / D.Hkv) > 1 << 30) return false;
  *p = kv_plan(D.bf16, n_seqs, n_rows, max_rows, (int64_t)max_pages * page_len, D.H, D.Hkv, D.dh);
  return kv_grid(*p, D.Hkv) <= kMaxBlocks && ((int64_t)n_rows * D.H + 3) / 4 <= kMaxBlocks;
}

bool ranges_meet(const void* a, int64_t la, const void* b, int64_t lb) {
  return (uintptr_t)a < (uintptr_t)b + lb && (uintptr_t)b < (uintptr_t)a + la;
}

// Whether two sets of n rows may share memory (rows of equal stride may lie between each other).
bool rows_meet(const char* a, int64_t sa, int64_t la, const char* b, int64_t sb, int64_t lb, int64_t n) {
  const intptr_t d = (intptr_t)b - (intptr_t)a;
  if (d >= (n - 1) * sa + la || -d >= (n - 1) * sb + lb) return false;
  if (sa != sb) return true;
  const int64_t m = ((int64_t)d % sa + sa) % sa;
  return !(m >= la && m + lb <= sa);
}

}  // namespace

extern "C" {

armt_status armt_kv_append(const armt_config* cfg, const armt_kv_cache* cache, const void* qkv, int64_t ld_qkv, int32_t n_rows,
                           const int32_t* positions, void* q_out, void* hip_stream) {
  Dims D;
  KvView v;
  ARMT_TRY(check_cache(cfg, cache, n_rows, &D, &v));
  if (!qkv || !q_out) return ARMT_ERR_NULL;
  if (ld_qkv < D.Nqkv) return ARMT_ERR_SHAPE;
  if (ld_qkv * (int64_t)D.esz % 16 || (uintptr_t)qkv % 16 || (uintptr_t)q_out % 16) return ARMT_ERR_UNSUPPORTED;
  if (((int64_t)n_rows + KV_ROWS - 1) / KV_ROWS > kMaxBlocks) return ARMT_ERR_UNSUPPORTED;
  const int64_t esz = D.esz;
  if (ranges_meet(q_out, (int64_t)n_rows * D.H * D.dh * esz, qkv, ((int64_t)(n_rows - 1) * ld_qkv + D.Nqkv) * esz)) return ARMT_ERR_SHAPE;
  HIP_TRY(launch_kv_append(D.bf16, qkv, ld_qkv, v, positions, q_out, cache->k, cache->v, D.H, D.Hkv, D.dh, D.rope_theta, (hipStream_t)hip_stream));
  return ARMT_OK;
}

size_t armt_kv_attention_workspace_bytes(const armt_config* cfg, int32_t n_seqs, int32_t max_pages, int32_t page_len, int32_t n_rows, int32_t max_rows) {
  Dims D;
  KvPlan p;
  if (check_config(cfg, &D) != ARMT_OK || n_seqs < 1 || n_seqs > kMaxSeqs || max_pages < 1 || page_len < 1 || n_rows < 1 || max_rows < 1 ||
      !attention_plan(D, n_seqs, max_pages, page_len, n_rows, max_rows, &p))
    return 0;
  return p.total > kAlign ? p.total : kAlign;
}

armt_status armt_kv_attention(const armt_config* cfg, const armt_kv_cache* cache, const void* q, int32_t n_rows, int32_t max_rows,
                              const uint64_t* tree, void* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Dims D;
  KvView v;
  KvPlan p;
  ARMT_TRY(check_cache(cfg, cache, n_rows, &D, &v));
  if (!q || !out) return ARMT_ERR_NULL;
  if (max_rows < 1 || (tree && max_rows > 64)) return ARMT_ERR_SHAPE;
  if ((uintptr_t)q % 16 || (uintptr_t)out % 16) return ARMT_ERR_UNSUPPORTED;
  const int64_t bytes = (int64_t)n_rows * D.H * D.dh * (int64_t)D.esz;
  if (ranges_meet(q, bytes, out, bytes)) return ARMT_ERR_SHAPE;
  if (!attention_plan(D, cache->n_seqs, cache->max_pages, cache->page_len, n_rows, max_rows, &p)) return ARMT_ERR_UNSUPPORTED;
  if (!workspace || ((uintptr_t)workspace % kAlign) != 0 || workspace_bytes < std::max(p.total, kAlign)) return ARMT_ERR_WORKSPACE;
  HIP_TRY(launch_kv_attention(D.bf16, p, q, cache->k, cache->v, (const unsigned long long*)tree, v, out, (char*)workspace, D.H, D.Hkv, D.dh, max_rows,
                              (hipStream_t)hip_stream));
  return ARMT_OK;
}

size_t armt_beam_select_workspace_bytes(int32_t n_seqs, int32_t n_beams, int32_t vocab, int32_t n_out) {
  if (n_seqs < 1 || n_beams < 1 || vocab < 1 || n_out < 1 || n_out > BS_MAX || n_beams > BS_BEAMS || (int64_t)n_beams * vocab < n_out ||
      (int64_t)n_beams * vocab > 0x7fff0000 || (int64_t)n_seqs * n_beams > 0xffffff)
    return 0;
  if ((int64_t)n_seqs * n_beams * beam_parts((int64_t)n_seqs * n_beams, vocab) > kMaxBlocks || n_seqs > kMaxBlocks / 2) return 0;
  return beam_workspace((int64_t)n_seqs * n_beams, vocab, n_out);
}

armt_status armt_beam_select(const float* logits, int64_t ld_logits, const float* scores, int32_t n_seqs, int32_t n_beams, int32_t vocab, int32_t n_out,
                             float* out_scores, int32_t* out_parents, int32_t* out_tokens, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!logits || !scores || !out_scores || !out_parents || !out_tokens) return ARMT_ERR_NULL;
  if (n_seqs < 1 || n_beams < 1 || vocab < 1 || n_out < 1 || ld_logits < vocab || (int64_t)n_beams * vocab < n_out) return ARMT_ERR_SHAPE;
  const size_t need = armt_beam_select_workspace_bytes(n_seqs, n_beams, vocab, n_out);
  if (!need) return ARMT_ERR_UNSUPPORTED;
  if (!workspace || ((uintptr_t)workspace % kAlign) != 0 || workspace_bytes < need) return ARMT_ERR_WORKSPACE;
  const int64_t in = (int64_t)n_seqs * n_beams * 4, out = (int64_t)n_seqs * n_out * 4;
  if (ranges_meet(out_scores, out, scores, in) && !((const float*)out_scores == scores && n_out == n_beams)) return ARMT_ERR_SHAPE;
  if (ranges_meet(out_parents, out, scores, in) || ranges_meet(out_tokens, out, scores, in)) return ARMT_ERR_SHAPE;
  HIP_TRY(launch_beam_select(logits, ld_logits, scores, n_seqs, n_beams, vocab, n_out, out_scores, out_parents, out_tokens, (char*)workspace,
                             (hipStream_t)hip_stream));
  return ARMT_OK;
}

armt_status armt_beam_reorder(const int32_t* parents, int32_t n_seqs, int32_t n_beams, const armt_beam_state* states, int32_t n_states, void* hip_stream) {
  if (!parents || !states) return ARMT_ERR_NULL;
  if (n_seqs < 1 || n_beams < 1 || n_states < 1) return ARMT_ERR_SHAPE;
  if (n_beams > BS_BEAMS || n_states > BR_STATES) return ARMT_ERR_UNSUPPORTED;
  BeamStates st{};
  const int64_t rows = (int64_t)n_seqs * n_beams;
  for (int i = 0; i < n_states; ++i) {
    const armt_beam_state& s = states[i];
    if (!s.src || !s.dst) return ARMT_ERR_NULL;
    if (s.row_bytes < 1 || s.row_bytes > (int64_t)1 << 40) return ARMT_ERR_SHAPE;
    const int64_t a = s.src_stride ? s.src_stride : s.row_bytes, b = s.dst_stride ? s.dst_stride : s.row_bytes;
    if (a < s.row_bytes || b < s.row_bytes || a > (int64_t)1 << 40 || b > (int64_t)1 << 40) return ARMT_ERR_SHAPE;
    st.s[i] = BeamState{(const char*)s.src, (char*)s.dst, s.row_bytes, a, b, 0, 0};
  }
  // what one state writes may be read only as its own source, row for row
  for (int i = 0; i < n_states; ++i)
    for (int j = 0; j < n_states; ++j) {
      const BeamState &d = st.s[i], &s = st.s[j];
      const bool in_place = i == j && d.src == d.dst && d.src_stride == d.dst_stride;
      if (!in_place && rows_meet(d.dst, d.dst_stride, d.row_bytes, s.src, s.src_stride, s.row_bytes, rows)) return ARMT_ERR_SHAPE;
      if (i != j && rows_meet(d.dst, d.dst_stride, d.row_bytes, s.dst, s.dst_stride, s.row_bytes, rows)) return ARMT_ERR_SHAPE;
    }
  st.n = n_states;
  const int unit = beam_reorder_unit(st, n_beams);
  const int64_t blocks = beam_reorder_blocks(st, n_seqs, unit);
  if (blocks < 1) return ARMT_ERR_UNSUPPORTED;
  HIP_TRY(launch_beam_reorder(st, blocks, unit, parents, n_beams, (hipStream_t)hip_stream));
  return ARMT_OK;
}

}  // extern "C"
