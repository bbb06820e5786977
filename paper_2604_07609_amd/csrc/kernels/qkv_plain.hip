// QKV projection of models whose rotation and KV write are a kernel of their own
#include "../phase_kernels.h"

PHASE_KERNEL8(k_qkv_plain, PH_QKV_PLAIN)
