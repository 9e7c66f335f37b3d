// Instantiations of attention over listed blocks: 4-bit codes, rows of up to 128 numbers.
#include "pag_kv_blocks.h"

template void pagkv::launch_blocks<PAG_KV_FP4, 2>(hipStream_t, const pagkv::Attend&, int, bool);
