#define BIQ_ATTEND_TYPE BIQ_F32
#define BIQ_ATTEND_LAUNCH launch_attend_f32
#include "biq_launch_attend.inc"
