// Many query rows over e5m2 caches.
#include "kvx_attend_rows.h"

namespace kvx {
template int launch_rows<kCodesE5m2>(const AttendArgs&, const AttendPlan&, int, void*);
}  // namespace kvx
