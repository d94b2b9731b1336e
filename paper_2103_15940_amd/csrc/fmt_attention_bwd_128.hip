// Attention, backward: heads of at most 128 columns, of more than 64.
#include "fmt_attention_bwd.h"

namespace fmt {
template void run_attention_bwd<4>(const AttnBwd &, bool, bool, dim3, hipStream_t);
}  // namespace fmt
