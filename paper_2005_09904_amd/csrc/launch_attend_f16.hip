#define BIQ_ATTEND_TYPE BIQ_F16
#define BIQ_ATTEND_LAUNCH launch_attend_f16
#include "biq_launch_attend.inc"
