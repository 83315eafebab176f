// The kernel for few query rows with up to 48 rows to a workgroup: for the commonest record layout alone (chunk_few_rows).
#include "chunk_few.h"

namespace mixkvq {
hipError_t start_chunk_few_3(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) { return few::start<3, 4, 0, 1>(a, c, units, s); }
}  // namespace mixkvq
