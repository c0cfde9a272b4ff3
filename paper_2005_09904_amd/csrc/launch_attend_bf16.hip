#define BIQ_ATTEND_TYPE BIQ_BF16
#define BIQ_ATTEND_LAUNCH launch_attend_bf16
#include "biq_launch_attend.inc"
