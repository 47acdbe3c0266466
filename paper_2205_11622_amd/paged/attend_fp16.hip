#include "attend_launch.hpp"

namespace slnr {
namespace paged {

int attend_fp16(const Launch &l, const AttendArgs &a, int64_t max_new) { return attend_type<_Float16>(l, a, max_new); }

}  // namespace paged
}  // namespace slnr
