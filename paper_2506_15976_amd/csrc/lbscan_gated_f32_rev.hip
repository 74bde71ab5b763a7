// Gated linear recurrence: fp32 storage, rows scanned from their end.
#define LBSCAN_GATED_T float
#define LBSCAN_GATED_REVERSE true
#define LBSCAN_GATED_LAUNCH launch_gated_f32_rev
#include "lbscan_gated.inc"
