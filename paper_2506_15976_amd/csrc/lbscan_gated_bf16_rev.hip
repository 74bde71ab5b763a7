// Gated linear recurrence: bf16 storage, rows scanned from their end.
#define LBSCAN_GATED_T bf16_t
#define LBSCAN_GATED_REVERSE true
#define LBSCAN_GATED_LAUNCH launch_gated_bf16_rev
#include "lbscan_gated.inc"
