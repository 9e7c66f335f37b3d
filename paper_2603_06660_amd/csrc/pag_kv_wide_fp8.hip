// Instantiations of the attention kernels for many query rows: 8-bit float codes.
#include "pag_kv_wide.h"

template int pagkv::launch_wide<PAG_KV_FP8>(hipStream_t, const pagkv::Attend&, int);
