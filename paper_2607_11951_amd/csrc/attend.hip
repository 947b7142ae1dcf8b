// attend.hip -- grid_attend: attention of a chunk of new tokens over a paged cache (gfx950).  The kernels: attend.h.
#include "attend.h"

using namespace grid;

extern "C" size_t grid_attend_workspace_bytes(const grid_paged_cache* cache, const grid_chunks* chunks,
                                              const grid_attend_args* args) {
  if (check("grid_attend", cache, chunks, args, false) != GRID_OK) return 0;
  return workspace_of(cache, chunks, shape_of(cache, chunks, args));
}

extern "C" int grid_attend(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_attend_args* args,
                           void* stream) {
  clear_error();
  const int rc = check("grid_attend", cache, chunks, args, true);
  if (rc != GRID_OK || chunks->n_tokens == 0) return rc;
  return attend<false>("grid_attend", cache, chunks, args, nullptr, stream);
}
