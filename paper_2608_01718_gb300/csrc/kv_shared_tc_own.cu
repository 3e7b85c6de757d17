// The attention kernel for many rows: its pass over each sequence's own positions, joined with the common part.
#define LC_TC_FORM kOwn
#define LC_TC_LAUNCH launch_own_tc
#include "kv_attend_tc.cu"
