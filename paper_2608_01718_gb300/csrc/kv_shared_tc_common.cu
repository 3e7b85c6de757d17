// The attention kernel for many rows: its pass over what groups of sequences have in common.
#define LC_TC_FORM kCommon
#define LC_TC_LAUNCH launch_common_tc
#include "kv_attend_tc.cu"
