// Many query rows over 16-bit caches.
#include "kvx_attend_rows.h"

namespace kvx {
template int launch_rows<kCodes16>(const AttendArgs&, const AttendPlan&, int, void*);
}  // namespace kvx
