#define BIQ_ATTEND_TYPE BIQ_F32
#define BIQ_ATTEND_LAUNCH launch_attend_shared_f32
#define BIQ_ATTEND_JOIN launch_shared_join_f32
#include "biq_launch_attend_shared.inc"
