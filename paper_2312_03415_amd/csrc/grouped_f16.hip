#define RL_T _Float16
#define RL_GROUPED_FN grouped_launch_f16
#define RL_GROUPED_ROWS_FN grouped_rows_launch_f16
#define RL_GROUPED_GRADS_FN grouped_grads_launch_f16
#include "grouped_launch.inc"
