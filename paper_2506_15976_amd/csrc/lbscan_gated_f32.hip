// Gated linear recurrence: fp32 storage, rows scanned from their start.
#define LBSCAN_GATED_T float
#define LBSCAN_GATED_REVERSE false
#define LBSCAN_GATED_LAUNCH launch_gated_f32
#include "lbscan_gated.inc"
