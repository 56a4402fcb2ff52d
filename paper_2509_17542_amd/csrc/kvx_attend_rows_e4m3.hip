// Many query rows over e4m3fn caches.
#include "kvx_attend_rows.h"

namespace kvx {
template int launch_rows<kCodesE4m3>(const AttendArgs&, const AttendPlan&, int, void*);
}  // namespace kvx
