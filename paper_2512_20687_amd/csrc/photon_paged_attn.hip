// Attention over a paged K/V cache: splits, the merge of their results, the C ABI.
#include "photon_paged_attn.h"

namespace photon {
namespace {

// Workgroups over the entries of a stream: as many as the chip holds at once (two a unit; one where a workgroup's registers fill it), but
// none with less than a step a wave (wide: eight steps, which all waves take), and none where that leaves fewer than eight: the merge is a launch.
// Microseconds, with 1, 2, 4, 8, 16 workgroups, the rule's marked:
//   one row, 16 streams of 2048 entries of 64     fp32 33.6, 22.7, 15.7, 12.2, 10.7*      bf16 15.6, 13.5, 10.9, 9.8, 9.6*
//   one row, 16 streams of 1024 of 64             fp32 17.8, 14.6, 11.5, 10.4*, 9.8       bf16 10.0, 10.9, 9.7, 9.4*, 9.8
//   one row, 64 streams of 2048 of 64             fp32 35.0, 23.7, 18.2, 18.5*, 21.0      bf16 18.7, 15.3, 12.8, 12.8*, 13.4
//   one row, 16 and 64 streams of 600 of 64       bf16 9.1*, 11.4, 10.7, 10.2, 9.9 and 9.0*, 11.0, 10.5, 11.2, 11.2; fp32 13.1*, 13.2, 11.6, 10.6, 9.8
//   one row, 32 streams of 32749 of 128           bf16 414, 220, 125, 99, 100*
//   20 rows, 8 streams of 3000 of 128             bf16 -, -, 21.6, 18.1, 16.8; 23 workgroups* 16.7
//   256 rows, 128 streams of 4096 of 128          wide 214, 146*, 165
//   2048 rows, 16 streams of 8191 of 128          wide 395, 236*, 251
int paged_auto_splits(int Bt, int T, int H, int H_kv, int d_p, int64_t S_max, bool f32_rows, photon_dtype kv_dt) {
  const int64_t rows = (int64_t)T * (H / H_kv);
  const PagedTile tile = paged_tile(rows, (int64_t)Bt * H_kv, f32_rows, kv_dt);
  const int64_t groups = (int64_t)Bt * H_kv * ((rows + tile.rows() - 1) / tile.rows());
  const int64_t steps = (S_max + PAGED_STEP - 1) / PAGED_STEP;
  int64_t splits = (tile.tiles == 1 ? 512 : 256) / groups;
  // Two tiles a wave leave more to merge: their second workgroup a unit has to have 16 steps a wave (64 rows over 128 streams of 2000, 4000
  // and 8000 entries of 128, with one split and with two: E4M3 pages 30.6 and 33.1, 55.5 and 51.0, 116 and 87 us; bf16 37.8 and 40.4, 73.9
  // and 69.2, 133 and 119).
  const bool held = tile.tiles == 2 && !tile.wide && paged_two_waves(d_p, 2, f32_rows || kv_dt == PHOTON_F32);
  if (held && steps * tile.waves / PAGED_WAVES / 16 >= 512 / groups) splits = 512 / groups;
  const int64_t most = tile.wide ? steps / 8 : steps * tile.waves / PAGED_WAVES;
  splits = splits > most ? most : splits;
  if (!tile.wide && most < 8) splits = 1;
  return (int)(splits < 1 ? 1 : splits > 256 ? 256 : splits);
}
int paged_most_splits(const photon_paged_cache* c, int Bt, int T, int H, int64_t S_max) {   // of either dtype of rows
  const int d_p = kv_row_elems(c->d_h);
  const int a = paged_auto_splits(Bt, T, H, c->H_kv, d_p, S_max, false, c->kv_dt), b = paged_auto_splits(Bt, T, H, c->H_kv, d_p, S_max, true, c->kv_dt);
  return a > b ? a : b;
}

constexpr int MANY_SPLITS = 9;            // from which on a row's are merged by all lanes of a workgroup

template <typename T, int NB> int32_t launch_merge(const PagedAttnArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.Bt * a.T * a.H;
  constexpr int per = 256 / (8 * NB);
  if (a.n_splits >= MANY_SPLITS && rows <= (int64_t)0xffffffff / 256) PHOTON_LAUNCH(KC_COARSE_MERGE, st, (paged_merge_kernel<T, NB, per>), dim3((unsigned)rows), dim3(256), 0, st, a);
  else PHOTON_LAUNCH(KC_COARSE_MERGE, st, (paged_merge_kernel<T, NB, 1>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, a);
  return check_launch("paged_merge_kernel");
}
template <typename T> int32_t launch_merge_t(const PagedAttnArgs& a, hipStream_t st) {
  const int nb = kv_row_elems(a.pool.d_h) / 32;
  return nb == 1 ? launch_merge<T, 1>(a, st) : nb == 2 ? launch_merge<T, 2>(a, st) : launch_merge<T, 4>(a, st);
}

// What the two entry points refuse of a shape.
int32_t check_queries(const char* who, const photon_paged_cache* c, int32_t Bt, int32_t T, int32_t H, int64_t S_max, int32_t n_splits) {
  PHOTON_REQUIRE(H > 0 && H % c->H_kv == 0, PHOTON_ERR_INVALID_ARG, "%s: H=%d query heads do not share H_kv=%d evenly", who, H, c->H_kv);
  PHOTON_REQUIRE(S_max > 0 && S_max <= (int64_t)c->max_pages * c->page_size, PHOTON_ERR_INVALID_ARG, "%s: S_max=%lld is not in [1, %d pages of %d]", who,
                 (long long)S_max, c->max_pages, c->page_size);
  PHOTON_REQUIRE(n_splits >= 0 && n_splits <= 1024, PHOTON_ERR_INVALID_ARG, "%s: n_splits=%d out of [0, 1024]", who, n_splits);
  PHOTON_REQUIRE(T <= 65535 && H <= 65535, PHOTON_ERR_UNSUPPORTED, "%s: T=%d, H=%d queries: at most 65535 each", who, T, H);
  return PHOTON_OK;
}

size_t workspace_bytes_of(const photon_paged_cache* c, int32_t Bt, int32_t T, int32_t H, int n_splits) {
  return n_splits <= 1 ? 0 : (size_t)Bt * T * H * n_splits * (kv_row_elems(c->d_h) + 2) * sizeof(float);
}

}  // namespace
}  // namespace photon

// ------------------------------------------------------------------ C ABI

using namespace photon;

extern "C" size_t photon_paged_attn_workspace_bytes(const photon_paged_cache* cache, int32_t Bt, int32_t T, int32_t H, int64_t S_max, int32_t n_splits) {
  if (cache == nullptr || cache->H_kv <= 0 || Bt <= 0 || T <= 0 || H < cache->H_kv || S_max <= 0 || kv_row_elems(cache->d_h) == 0) return 0;
  return workspace_bytes_of(cache, Bt, T, H, n_splits == 0 ? paged_most_splits(cache, Bt, T, H, S_max) : n_splits);
}

extern "C" int32_t photon_paged_attn(const photon_paged_cache* cache, const void* q, int64_t q_stride, const int32_t* seq_len, const int32_t* n_new,
                                     const uint64_t* tree, void* out, int32_t* status, int32_t Bt, int32_t T, int32_t H, int64_t S_max, float scale,
                                     int32_t n_splits, void* workspace, size_t workspace_bytes, photon_dtype dt, void* stream) {
  clear_error();
  PagedAttnArgs a;
  PHOTON_TRY(paged_pools(__func__, cache, Bt, T, &a.pool));
  PHOTON_REQUIRE(valid_dtype(dt), PHOTON_ERR_UNSUPPORTED, "%s: rows are fp32 or bf16, not dtype %d", __func__, (int)dt);
  PHOTON_TRY(check_queries(__func__, cache, Bt, T, H, S_max, n_splits));
  PHOTON_REQUIRE(tree == nullptr || T <= PAGED_MOST_TREE, PHOTON_ERR_UNSUPPORTED, "%s: a tree of T=%d nodes: at most %d", __func__, T, PAGED_MOST_TREE);
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const size_t esz = dtype_size(dt);
  const int d_h = cache->d_h;
  PHOTON_REQUIRE(q && out && element_aligned(q, esz) && element_aligned(out, esz), PHOTON_ERR_INVALID_ARG, "%s: q and out must be non-null device pointers to whole elements", __func__);
  PHOTON_REQUIRE(seq_len != nullptr, PHOTON_ERR_INVALID_ARG, "%s: seq_len is null", __func__);
  PHOTON_REQUIRE(q_stride >= (int64_t)H * d_h, PHOTON_ERR_INVALID_ARG, "%s: q_stride=%lld is less than a row of %d heads of %d", __func__, (long long)q_stride, H, d_h);
  const bool f32 = dt == PHOTON_F32;
  if (n_splits == 0) n_splits = paged_auto_splits(Bt, T, H, cache->H_kv, kv_row_elems(d_h), S_max, f32, cache->kv_dt);
  if (n_splits > 1) {
    const size_t need = workspace_bytes_of(cache, Bt, T, H, n_splits);
    PHOTON_REQUIRE(workspace != nullptr && aligned16(workspace) && workspace_bytes >= need, PHOTON_ERR_WORKSPACE,
                   "%s: n_splits=%d needs a 16-byte aligned workspace of %zu bytes (got %zu)", __func__, n_splits, need, workspace_bytes);
  }
  a.q = q; a.out = out; a.ws = (float*)workspace;
  a.seq_len = seq_len; a.n_new = n_new; a.tree = tree; a.status = status;
  a.q_stride = q_stride; a.S_max = (int32_t)S_max; a.Bt = Bt; a.T = T; a.H = H; a.group = H / cache->H_kv; a.n_splits = n_splits;
  const int64_t rows = (int64_t)T * a.group;
  const PagedTile tile = paged_tile(rows, (int64_t)Bt * cache->H_kv, f32, cache->kv_dt);
  PHOTON_REQUIRE(rows <= PAGED_MOST_ROWS, PHOTON_ERR_UNSUPPORTED, "%s: T=%d queries of %d heads a K/V head are too many", __func__, T, a.group);
  const int64_t groups = (rows + tile.rows() - 1) / tile.rows(), units = (int64_t)Bt * cache->H_kv * n_splits;
  PHOTON_REQUIRE((units + 7) * groups <= (int64_t)0xffffffff / 512 && (int64_t)Bt * T * H <= (int64_t)0xffffffff / 32, PHOTON_ERR_UNSUPPORTED,
                 "%s: Bt=%d, T=%d, H=%d, n_splits=%d are too many workgroups", __func__, Bt, T, H, n_splits);
  a.row_groups = (int32_t)groups; a.units = (int32_t)units;
  a.half_scale = scale * (0.5f * LOG2E);
  a.q_pieces = d_h % 4 == 0 && q_stride % 4 == 0 && element_aligned(q, 4 * esz);
  a.out_pieces = d_h % 4 == 0 && element_aligned(out, 4 * esz);
  hipStream_t st = (hipStream_t)stream;
  switch (cache->kv_dt) {
    case PHOTON_F32: PHOTON_TRY(paged_attn_f32(a, tile, f32, st)); break;
    case PHOTON_BF16: PHOTON_TRY(paged_attn_bf16(a, tile, f32, st)); break;
    default: PHOTON_TRY(paged_attn_e4m3(a, tile, f32, st)); break;
  }
  if (n_splits == 1) return PHOTON_OK;
  return f32 ? launch_merge_t<float>(a, st) : launch_merge_t<bf16_t>(a, st);
}
