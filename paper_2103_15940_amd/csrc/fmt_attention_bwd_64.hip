// Attention, backward: heads of at most 64 columns.
#include "fmt_attention_bwd.h"

namespace fmt {
template void run_attention_bwd<2>(const AttnBwd &, bool, bool, dim3, hipStream_t);
}  // namespace fmt
