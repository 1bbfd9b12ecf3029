// Attention over memories whose first pages are packed, or of which rows see a span.
#pragma once

#include "packed.h"

namespace cs {

struct SpanJob {
  const int32_t* blocks;  // DEVICE [B] packed pages of every request, or null
  int sinks, window;
};
size_t packed_attend_workspace(const Geo& g);
// (packed is null where job.blocks is)
cs_status launch_packed_attend(const Geo& g, const cs_page_pool& pool, const cs_packed_pool* packed, int layer,
                               const cs_batch& b, const SpanJob& job, const cs_rows& q, const cs_rows& out, float* lse,
                               void* ws, hipStream_t s, bool check_only);

}  // namespace cs
