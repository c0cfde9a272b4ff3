#define BIQ_ATTEND_TYPE BIQ_BF16
#define BIQ_ATTEND_LAUNCH launch_attend_shared_bf16
#define BIQ_ATTEND_JOIN launch_shared_join_bf16
#include "biq_launch_attend_shared.inc"
