// What the host entry points that take a paged cache share.  Defined in api_paged.cu.
#pragma once

#include "../../include/s2a.h"
#include "paged.h"

namespace s2a {

int check_cache(const s2a_cache* c);
int check_batch(const s2a_batch* b, const s2a_cache* c);
int check_heads(const s2a_cache* cache, const s2a_batch* batch, int H, int max_new, int window, int sinks);
PagedBatch batch_of(const s2a_batch* b);
PagedPool pool_of(const s2a_cache* c);

}  // namespace s2a
