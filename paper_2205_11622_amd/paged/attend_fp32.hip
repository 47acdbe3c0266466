#include "attend_launch.hpp"

namespace slnr {
namespace paged {

int attend_fp32(const Launch &l, const AttendArgs &a, int64_t max_new) { return attend_type<float>(l, a, max_new); }

}  // namespace paged
}  // namespace slnr
