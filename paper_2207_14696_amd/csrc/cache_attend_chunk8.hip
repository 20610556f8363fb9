// the kernel for many rows, codes of 8 bits
#include "cache_attend_chunk_launch.hpp"

namespace bf {
template hipError_t attend_chunk_bits<8>(const AttendCall &, const AttendPlan &, int);
}  // namespace bf
