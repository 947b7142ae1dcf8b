// attend_tree.hip -- grid_attend_tree: attention of trees of drafted tokens over a paged cache (gfx950).  The kernels:
// attend.h.
#include "attend.h"

using namespace grid;

extern "C" size_t grid_attend_tree_workspace_bytes(const grid_paged_cache* cache, const grid_chunks* chunks,
                                                   const grid_attend_args* args) {
  if (check("grid_attend_tree", cache, chunks, args, false) != GRID_OK) return 0;
  return workspace_of(cache, chunks, shape_of(cache, chunks, args, true));
}

extern "C" int grid_attend_tree(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_attend_args* args,
                                const grid_tree* tree, void* stream) {
  clear_error();
  const int rc = check("grid_attend_tree", cache, chunks, args, true);
  if (rc != GRID_OK) return rc;
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_attend_tree: ") + what); };
  if (!tree) return bad("null argument");
  const int64_t words = ((int64_t)std::min(args->max_q, chunks->n_tokens) + 31) / 32;
  if (tree->stride_words < words || tree->stride_words > INT32_MAX) return bad("fewer mask words than a chunk has tokens");
  if (chunks->n_tokens == 0) return GRID_OK;
  if (!tree->masks || (uintptr_t)tree->masks % 4 != 0) return bad("no masks");
  if (args->window && !tree->depth) return bad("a window asks for depths");
  return attend<true>("grid_attend_tree", cache, chunks, args, tree, stream);
}
