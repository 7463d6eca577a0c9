#define RL_T __bf16
#define RL_GROUPED_FN grouped_launch_bf16
#define RL_GROUPED_ROWS_FN grouped_rows_launch_bf16
#define RL_GROUPED_GRADS_FN grouped_grads_launch_bf16
#include "grouped_launch.inc"
