// Instantiations of attention over listed blocks: 8-bit float codes, rows of up to 256 numbers.
#include "pag_kv_blocks.h"

template void pagkv::launch_blocks<PAG_KV_FP8, 4>(hipStream_t, const pagkv::Attend&, int, bool);
