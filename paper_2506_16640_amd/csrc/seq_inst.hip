// One translation unit per (element type, head dimension) of the serving attention: -DENTMAX_INST_T=<bf16_t|float>, -DENTMAX_INST_D=<64|128>
#include "seq_run.hip.h"
namespace entmax {
template int run_seq<ENTMAX_INST_T, ENTMAX_INST_D>(const SeqCall&);
}
