"""B200-native MI hook: CUDA kernels behind a C ABI (include/mix.h) plus a thin binding."""
from .binding import *          # noqa: F401,F403
from .binding import Mix, MixError, load_library, set_pdl_mask  # noqa: F401
from .experts import (expert_combine, expert_combine_grad, expert_order, linear_int, linear_int_grouped, linear_int_status, quantize_rows,  # noqa: F401
                      router_balance, router_balance_grad, router_topk, router_topk_grad)
