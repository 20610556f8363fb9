// the kernel for many rows, codes of 4 bits
#include "cache_attend_chunk_launch.hpp"

namespace bf {
template hipError_t attend_chunk_bits<4>(const AttendCall &, const AttendPlan &, int);
}  // namespace bf
