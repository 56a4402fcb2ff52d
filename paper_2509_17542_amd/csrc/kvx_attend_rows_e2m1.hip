// Many query rows over 4-bit e2m1 caches.
#include "kvx_attend_rows.h"

namespace kvx {
template int launch_rows<kCodesE2m1>(const AttendArgs&, const AttendPlan&, int, void*);
}  // namespace kvx
