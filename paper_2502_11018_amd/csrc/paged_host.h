// Checks and conversions of the paged cache's descriptors, shared by its own
// entry points and by the verify contexts that use such a cache.
#pragma once

#include "griffin_verify.h"
#include "paged.h"

namespace griffin {

int paged_pool_of(const griffin_pool& p, PagedPool* out);
int paged_table_of(const griffin_pool& pool, const int32_t* table, int stride, int cols, const int32_t* lengths,
                   int max_length, PagedTable* out);
// whether the rows and workgroups of such calls can be counted and launched
bool paged_sizes(const PagedPool& pool, int batch, int nodes, int n_q_heads);
void paged_frequencies(double base, int dh, double* inv_rev);

}  // namespace griffin
