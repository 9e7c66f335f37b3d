// Instantiations of the attention kernels for few query rows: 4-bit codes, rows of up to 256 numbers.
#include "pag_kv_narrow.h"

template void pagkv::launch_narrow<PAG_KV_FP4, 4>(hipStream_t, const pagkv::Attend&, int, bool);
