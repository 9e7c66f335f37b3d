// Instantiations of the attention kernels for many query rows: 8-bit integer codes.
#include "pag_kv_wide.h"

template int pagkv::launch_wide<PAG_KV_INT8>(hipStream_t, const pagkv::Attend&, int);
