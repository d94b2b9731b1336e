// Attention, forward: heads of at most 64 columns.
#include "fmt_attention_fwd.h"

namespace fmt {
template void run_attention_fwd<2>(const AttnFwd &, const FwdChoice &, dim3, hipStream_t);
}  // namespace fmt
