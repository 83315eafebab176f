// The kernel for few query rows with up to 16 rows to a workgroup.
#include "chunk_few.h"

namespace mixkvq {
hipError_t start_chunk_few_1(const CacheView& v, const ChunkArgs& a, const ChunkLaunch& l, bool split, hipStream_t s) {
  return few::start_any<1>(v, a, l, split, s);
}
}  // namespace mixkvq
