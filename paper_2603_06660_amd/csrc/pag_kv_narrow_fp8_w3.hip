// Instantiations of the attention kernels for few query rows: 8-bit float codes, rows of 136 to 192 numbers.
#include "pag_kv_narrow.h"

template void pagkv::launch_narrow<PAG_KV_FP8, 3>(hipStream_t, const pagkv::Attend&, int, bool);
