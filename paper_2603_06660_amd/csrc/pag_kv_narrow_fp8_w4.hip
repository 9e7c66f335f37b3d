// Instantiations of the attention kernels for few query rows: 8-bit float codes, rows of 200 to 256 numbers.
#include "pag_kv_narrow.h"

template void pagkv::launch_narrow<PAG_KV_FP8, 4>(hipStream_t, const pagkv::Attend&, int, bool);
