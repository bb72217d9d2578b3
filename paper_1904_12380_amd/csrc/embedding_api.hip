// C ABI of the embedding table: argument checks, workspace and launches.
// Declarations and contract: include/decoder_mi355x.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sm_decoder_host.hpp"
#include "sm_embedding.hpp"

namespace {

using namespace smx;
using namespace smx_host;

#define SMX_BY_TYPE(dtype, K)                                                        \
  ((dtype) == SOFTMAX_F32   ? reinterpret_cast<const void*>(&K<float>)               \
   : (dtype) == SOFTMAX_F16 ? reinterpret_cast<const void*>(&K<f16>)                 \
                            : reinterpret_cast<const void*>(&K<bf16>))
#define SMX_BY_GROUP(dtype, g, K)                                                    \
  ((dtype) == SOFTMAX_F32   ? by_group<float>(g, K)                                  \
   : (dtype) == SOFTMAX_F16 ? by_group<f16>(g, K) : by_group<bf16>(g, K))

constexpr int kSums = 0, kJoin = 1;

template <typename T, int G>
const void* of_group(int what) {
  return what == kSums ? reinterpret_cast<const void*>(&k_embed_sums<T, G>)
                       : reinterpret_cast<const void*>(&k_embed_join<T, G>);
}
template <typename T>
const void* by_group(int g, int what) {
  return g == 8 ? of_group<T, 8>(what) : g == 16 ? of_group<T, 16>(what)
         : g == 32 ? of_group<T, 32>(what) : of_group<T, 64>(what);
}

// Lanes that take a chunk's columns: as many as a row has strips, up to a
// wavefront.
int group_of(int64_t strips) { return strips <= 8 ? 8 : strips <= 16 ? 16 : strips <= 32 ? 32 : 64; }

// Sorted tokens of a chunk: 8, or so many more that the chunks' columns still make
// 4096 wavefronts, up to 32; and more once that makes 8192 chunks, which keeps the
// parts of a run that an id with many tokens has few.
int64_t chunk_of(int64_t tokens, int64_t strips) {
  const int64_t waves = ceil_div(tokens * strips, 64);
  const int64_t chunk = std::clamp<int64_t>(waves / 4096 / 8 * 8, 8, 32);
  return std::max(chunk, up_to(ceil_div(tokens, 8192), 8));
}

struct Room {
  int64_t key[2], token[2], bins, part, end;
  int64_t tiles, chunk, chunks;
};

Room room(int64_t tokens, int64_t d, int dtype) {
  Room r;
  const int64_t list = up_to(tokens * 4, 16);
  const bool radix = tokens > kMergeMost;
  r.chunk = chunk_of(tokens, d * dtype_size(dtype) / 16);
  r.chunks = ceil_div(tokens, r.chunk);
  r.tiles = ceil_div(tokens, radix ? kMoveTile : kTile);
  for (int i = 0; i < 2; ++i) {
    r.key[i] = 2 * i * list;
    r.token[i] = (2 * i + 1) * list;
  }
  r.bins = 4 * list;
  r.part = r.bins + (radix ? up_to(r.tiles * kBins * 4, 16) : 0);
  r.end = r.part + (r.chunks > 1 ? r.chunks * 2 * d * 4 : 0);
  return r;
}

bool sizes_ok(int64_t tokens, int64_t rows, int64_t d, int dtype) {
  return dtype_size(dtype) != 0 && count_ok(tokens) && count_ok(rows) && width_ok(d);
}

// Workgroups of a launch of `threads` threads for `units` threads of work; -1
// past what a launch takes.
int64_t groups(int64_t units, int threads) {
  const int64_t n = ceil_div(units, threads);
  return n < (int64_t(1) << 32) / threads ? n : -1;
}

hipError_t start(const void* fn, int64_t grid, int threads, void** args, hipStream_t s) {
  return launch(fn, grid, threads, args, s);
}

}  // namespace

extern "C" {

SOFTMAX_API int softmax_embedding_fwd(const int64_t* ids, int64_t tokens, const void* table,
                                      int64_t table_stride, int64_t rows, int64_t d, float scale,
                                      int dtype, void* out, hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t tb = 0;
  if (!sizes_ok(tokens, rows, d, dtype) || !std::isfinite(scale) || table_stride < 0 ||
      table_stride > SOFTMAX_MAX_ROW_STRIDE || !rows_ok(table, rows, table_stride, d, size, &tb) ||
      !aligned16(out))
    return SOFTMAX_ERR_INVALID_ARG;
  if (tokens == 0) return SOFTMAX_OK;
  const int64_t grid = groups(ceil_div(tokens * d * size / 16, 4), 256);
  if (grid < 0) return SOFTMAX_ERR_INVALID_ARG;
  const Range inputs[] = {{ids, tokens * 8}, {table, tb}};
  const Range outputs[] = {{out, tokens * d * size}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  EmbedArgs a = {};
  a.ids = ids;
  a.in = table;
  a.pitch = table_stride;
  a.out = out;
  a.tokens = static_cast<int>(tokens);
  a.rows = static_cast<int>(rows);
  a.d = static_cast<int>(d);
  a.scale = scale;
  void* args[] = {&a};
  const hipError_t e = start(SMX_BY_TYPE(dtype, k_embed_rows), grid, 256, args, stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

SOFTMAX_API int64_t softmax_embedding_bwd_workspace(int64_t tokens, int64_t rows, int64_t d,
                                                    int dtype) {
  if (!sizes_ok(tokens, rows, d, dtype)) return -1;
  return rows == 0 ? 0 : room(tokens, d, dtype).end;
}

SOFTMAX_API int softmax_embedding_bwd(const void* dout, int64_t dout_stride, const int64_t* ids,
                                      int64_t tokens, int64_t rows, int64_t d, float scale,
                                      int dtype, void* dtable, void* workspace,
                                      int64_t workspace_bytes, hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t db = 0;
  if (!sizes_ok(tokens, rows, d, dtype) || !std::isfinite(scale) || dout_stride < 0 ||
      !rows_ok(dout, tokens, dout_stride, d, size, &db) || !aligned16(dtable) ||
      !aligned16(workspace))
    return SOFTMAX_ERR_INVALID_ARG;
  if (rows == 0) return SOFTMAX_OK;
  const Room r = room(tokens, d, dtype);
  if (workspace_bytes < r.end) return SOFTMAX_ERR_INVALID_ARG;
  const int64_t strips = d * size / 16;
  const int g = group_of(strips);
  const int64_t grid = groups(r.chunks * ceil_div(strips, g) * g, 256);
  if (grid < 0) return SOFTMAX_ERR_INVALID_ARG;
  const Range inputs[] = {{dout, db}, {ids, tokens * 8}};
  const Range outputs[] = {{dtable, rows * d * size}, {workspace, r.end}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  char* const at = static_cast<char*>(workspace);
  EmbedArgs a = {};
  a.ids = ids;
  a.in = dout;
  a.pitch = dout_stride;
  a.out = dtable;
  a.tokens = static_cast<int>(tokens);
  a.rows = static_cast<int>(rows);
  a.d = static_cast<int>(d);
  a.scale = scale;
  for (int i = 0; i < 2; ++i) {
    a.key[i] = reinterpret_cast<unsigned*>(at + r.key[i]);
    a.token[i] = reinterpret_cast<int*>(at + r.token[i]);
  }
  a.bins = reinterpret_cast<int*>(at + r.bins);
  a.part = reinterpret_cast<float*>(at + r.part);
  a.tiles = static_cast<int>(r.tiles);
  a.chunk = static_cast<int>(r.chunk);
  a.chunks = static_cast<int>(r.chunks);
  a.clear = rows * d * size / 16;
  // Keys are 0 .. rows.
  int passes = 1;
  while (passes * kDigit < 31 && rows >> (passes * kDigit) != 0) ++passes;
  a.passes = passes;
  hipError_t e = hipSuccess;
  void* one[] = {&a};
  const int64_t clear = std::min<int64_t>(ceil_div(a.clear, 4 * kSortThreads), 2048);
  if (tokens <= kMergeMost) {
    int tiles = static_cast<int>(r.tiles), to = tiles > 1 ? 1 : 0;
    void* sort[] = {&a, &tiles, &to};
    e = start(reinterpret_cast<const void*>(&k_embed_sort<0>), tiles + clear, kSortThreads, sort,
              stream);
    void* merge[] = {&a, &tiles};
    if (e == hipSuccess && tiles > 1)
      e = start(reinterpret_cast<const void*>(&k_embed_merge<0>),
                ceil_div(tokens * kMergeLanes, kSortThreads), kSortThreads, merge, stream);
  } else {
    a.sorted = passes & 1;
    for (int p = 0; p < passes && e == hipSuccess; ++p) {
      void* two[] = {&a, &p};
      e = start(reinterpret_cast<const void*>(&k_embed_count<0>), r.tiles + (p == 0 ? clear : 0),
                kSortThreads, two, stream);
      if (e == hipSuccess)
        e = start(reinterpret_cast<const void*>(&k_embed_base<0>), 1, 1024, one, stream);
      if (e == hipSuccess)
        e = start(reinterpret_cast<const void*>(&k_embed_move<0>), r.tiles, kSortThreads, two,
                  stream);
    }
  }
  if (e == hipSuccess && tokens > 0)
    e = start(SMX_BY_GROUP(dtype, g, kSums), grid, 256, one, stream);
  if (e == hipSuccess && r.chunks > 1)
    e = start(SMX_BY_GROUP(dtype, g, kJoin), grid, 256, one, stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

}  // extern "C"
