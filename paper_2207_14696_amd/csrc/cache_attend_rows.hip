// the kernel for few rows: which of its forms
#include "cache_attend_rows_impl.hpp"

namespace bf {
namespace {

template <int BITS, int DP, int NP, int WP>
void by_mode(const AttendCall &a, const AttendPlan &p) {
    const int mode = mode_of(a);
    auto kernel = mode == kCapped  ? attend_rows_kernel<BITS, DP, NP, WP, kCapped>
                  : mode == kBiased ? attend_rows_kernel<BITS, DP, NP, WP, kBiased>
                                    : attend_rows_kernel<BITS, DP, NP, WP, kPlain>;
    if constexpr (NP == 1)
        if (mode == kCappedFirst) kernel = attend_rows_kernel<BITS, DP, NP, WP, kCappedFirst>;
    kernel<<<grid_of(p), 256, 0, a.s>>>(a, p);
}

template <int BITS, int DP>
void by_type(const AttendCall &a, const AttendPlan &p) {
    if (a.dtype == BIFEAT_F32) by_mode<BITS, DP, 2, 2>(a, p);
    else if (a.dtype == BIFEAT_F16) by_mode<BITS, DP, 1, 2>(a, p);
    else by_mode<BITS, DP, 1, 1>(a, p);
}

}  // namespace

void launch_attend_rows(const AttendCall &a, const AttendPlan &p, int bits, int dp) {
    if (bits == 8) dp == 64 ? by_type<8, 64>(a, p) : dp == 128 ? by_type<8, 128>(a, p) : by_type<8, 256>(a, p);
    else dp == 64 ? by_type<4, 64>(a, p) : dp == 128 ? by_type<4, 128>(a, p) : by_type<4, 256>(a, p);
}

}  // namespace bf
