#include "cache_attend_rows_impl.hpp"

namespace bf {
template <int BITS, int DP>
static void go(const AttendCall &a, const AttendPlan &p) {
    const int mode = a.softcap > 0.f ? 2 : a.slopes ? 1 : 0;
    auto kernel = a.dtype == BIFEAT_F32 ? mode == 0   ? attend_rows_kernel<BITS, DP, 2, 0>
                                          : mode == 1 ? attend_rows_kernel<BITS, DP, 2, 1>
                                                      : attend_rows_kernel<BITS, DP, 2, 2>
                  : mode == 0           ? attend_rows_kernel<BITS, DP, 1, 0>
                  : mode == 1           ? attend_rows_kernel<BITS, DP, 1, 1>
                                        : attend_rows_kernel<BITS, DP, 1, 2>;
    kernel<<<p.nw, 256, 0, a.s>>>(a, p);
}
void launch_attend_rows(const AttendCall &a, const AttendPlan &p, int bits, int dp) {
    if (bits == 8) dp == 64 ? go<8, 64>(a, p) : dp == 128 ? go<8, 128>(a, p) : go<8, 256>(a, p);
    else dp == 64 ? go<4, 64>(a, p) : dp == 128 ? go<4, 128>(a, p) : go<4, 256>(a, p);
}
}  // namespace bf
