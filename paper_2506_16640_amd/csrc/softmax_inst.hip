// One translation unit per (element type, head dimension) of the softmax attention: -DENTMAX_INST_T=<bf16_t|float>, -DENTMAX_INST_D=<64|128>
#include "softmax.hip.h"
namespace entmax {
template int run_softmax<ENTMAX_INST_T, ENTMAX_INST_D>(const SoftmaxCall&);
}
