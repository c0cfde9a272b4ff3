#define BIQ_ATTEND_TYPE BIQ_F16
#define BIQ_ATTEND_LAUNCH launch_attend_shared_f16
#define BIQ_ATTEND_JOIN launch_shared_join_f16
#include "biq_launch_attend_shared.inc"
