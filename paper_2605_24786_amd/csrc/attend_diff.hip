// The decode attention's kernels whose rows are subtracted in pairs (conf_kv_attend_diff): the matrix-core body for an even number of
// rows.
#include "attend_body.h"

namespace confkv {

AttendFn attend_diff_instance(AttendForm form, int D, int G, bool chan) {
#define CONFKV_CASE(g)                                                                                                       \
  if (G == g && D == 64 && !chan)                                                                                            \
    return form == kFormMfma    ? (AttendFn)attend_mfma_kernel<g, false, false, 64, false, false, true>                      \
           : form == kFormPaged ? (AttendFn)attend_mfma_kernel<g, false, false, 64, true, false, true>                       \
                                : (AttendFn)attend_mfma_kernel<g, false, true, 64, false, false, true>;                      \
  if (G == g && D == 128 && form == kFormPaged)                                                                              \
    return chan ? nullptr : (AttendFn)attend_mfma_kernel<g, false, false, 128, true, false, true>;                           \
  if (G == g && D == 128 && form == kFormMfma)                                                                               \
    return chan ? (AttendFn)attend_mfma_kernel<g, true, false, 128, false, false, true>                                      \
                : (AttendFn)attend_mfma_kernel<g, false, false, 128, false, false, true>;                                    \
  if (G == g && D == 128 && form == kFormMfmaSpill)                                                                          \
    return chan ? (AttendFn)attend_mfma_kernel<g, true, true, 128, false, false, true>                                       \
                : (AttendFn)attend_mfma_kernel<g, false, true, 128, false, false, true>;
  if (form == kFormValu || form == kFormValuSpill) return nullptr;
  CONFKV_CASE(2) CONFKV_CASE(4) CONFKV_CASE(6) CONFKV_CASE(8)
#undef CONFKV_CASE
  // sixteen rows: several tokens, or groups of more than eight heads
  if (G == kChunkRows && D == 128 && form == kFormMfma)
    return chan ? (AttendFn)attend_mfma_kernel<kChunkRows, true, false, 128, false, false, true>
                : (AttendFn)attend_mfma_kernel<kChunkRows, false, false, 128, false, false, true>;
  if (G == kChunkRows && D == 128 && form == kFormMfmaSpill)
    return chan ? (AttendFn)attend_mfma_kernel<kChunkRows, true, true, 128, false, false, true>
                : (AttendFn)attend_mfma_kernel<kChunkRows, false, true, 128, false, false, true>;
  return nullptr;
}

AttendFn attend_diff_finish(int D, int G) {
#define CONFKV_CASE(g)                                                                                                       \
  if (G == g) return D == 64 ? (AttendFn)attend_finish_kernel<128, g, 64, true> : (AttendFn)attend_finish_kernel<128, g, 128, true>;
  CONFKV_CASE(2) CONFKV_CASE(4) CONFKV_CASE(6) CONFKV_CASE(8)
#undef CONFKV_CASE
  return G == kChunkRows && D == 128 ? (AttendFn)attend_finish_kernel<128, kChunkRows, 128, true> : nullptr;
}

}  // namespace confkv
