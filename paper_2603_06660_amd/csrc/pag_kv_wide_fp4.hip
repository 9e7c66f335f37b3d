// Instantiations of the attention kernels for many query rows: 4-bit codes.
#include "pag_kv_wide.h"

template int pagkv::launch_wide<PAG_KV_FP4>(hipStream_t, const pagkv::Attend&, int);
