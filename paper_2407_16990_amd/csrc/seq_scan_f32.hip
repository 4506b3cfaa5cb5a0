// rh_state_scan of fp32 rows.
#include "seq_scan.h"

hipError_t scan_launch_f32(rh_ctx* ctx, scan_args& a, rh_status* failed) { return launch_scan<float>(ctx, a, failed); }
