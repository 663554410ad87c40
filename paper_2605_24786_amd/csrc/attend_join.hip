// The decode attention's kernels with a shared prefix's partial results taken in (conf_kv_attend_shared's second launch).
#include "attend_body.h"

namespace confkv {

AttendFn attend_shared_instance(AttendForm form, int D, int G, bool chan) { return attend_instance<true>(form, D, G, chan); }

}  // namespace confkv
