#include "attend_fp4_launch.hpp"

namespace slnr {
namespace paged {

int attend_fp4_bf16(const Launch &l, const AttendFp4Args &a, int64_t max_new) {
  return attend_fp4_type<__bf16>(l, a, max_new);
}

}  // namespace paged
}  // namespace slnr
