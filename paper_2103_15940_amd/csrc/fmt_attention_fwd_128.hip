// Attention, forward: heads of at most 128 columns, of more than 64.
#include "fmt_attention_fwd.h"

namespace fmt {
template void run_attention_fwd<4>(const AttnFwd &, const FwdChoice &, dim3, hipStream_t);
}  // namespace fmt
