// Instantiations of attention over listed blocks: 8-bit integer codes, rows of up to 256 numbers.
#include "pag_kv_blocks.h"

template void pagkv::launch_blocks<PAG_KV_INT8, 4>(hipStream_t, const pagkv::Attend&, int, bool);
