#include "attend_launch.hpp"

namespace slnr {
namespace paged {

int attend_bf16(const Launch &l, const AttendArgs &a, int64_t max_new) { return attend_type<__bf16>(l, a, max_new); }

}  // namespace paged
}  // namespace slnr
