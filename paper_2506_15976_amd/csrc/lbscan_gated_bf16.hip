// Gated linear recurrence: bf16 storage, rows scanned from their start.
#define LBSCAN_GATED_T bf16_t
#define LBSCAN_GATED_REVERSE false
#define LBSCAN_GATED_LAUNCH launch_gated_bf16
#include "lbscan_gated.inc"
