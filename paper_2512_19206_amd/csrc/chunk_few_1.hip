// The kernel for few query rows with up to 16 rows to a workgroup.
#include "chunk_few.h"

namespace mixkvq {
hipError_t start_chunk_few_1(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) { return few::start_any<1>(a, c, units, s); }
}  // namespace mixkvq
