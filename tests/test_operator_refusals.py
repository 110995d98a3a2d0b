"""What the operators without a context refuse, before anything reaches a device (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2607_22595_b200 as mix

INVALID, RANGE, UNSUPPORTED = -1, -2, -3
P = 4096                                                    # stands for a device pointer: a refused call looks at no memory
SMALL_NORMAL = dict(topk=[P, 0, 8, 4, 8, 2, 1, 1, None, P, P], topk_grad=[P, 0, 8, 4, 8, 2, 1, 1, P, P, P, P, 8],
                    order=[P, 8, 8, P, P, P, None, 0], balance=[P, 0, 8, P, 4, 8, 2, 1, None, 1, P, P, P, P, P, 1 << 20],
                    balance_grad=[P, 0, 8, P, 4, 8, 2, 1, None, 1, P, P, P, P, 8], quantize=[P, 1, 64, 4, None, 1, 4, 64, P, P],
                    linear=[P, P, 4, 64, P, P, 8, None, P, 1, 8], grouped=[P, P, 4, 64, P, P, 2, 8, P, None, P, 1, 8],
                    combine=[P, 1, 8, 8, P, P, 4, 2, 8, P, 8], combine_grad=[P, 1, 8, 8, P, P, 4, 2, 8, P, 8, P, P, 8])
FN = dict(topk="mix_router_topk", topk_grad="mix_router_topk_grad", order="mix_expert_order", balance="mix_router_balance",
          balance_grad="mix_router_balance_grad", quantize="mix_quantize_rows", linear="mix_linear_int", grouped="mix_linear_int_grouped",
          combine="mix_expert_combine", combine_grad="mix_expert_combine_grad")
REFUSED = [
    ("topk", {0: None}, INVALID), ("topk", {1: 3}, INVALID), ("topk", {2: 7}, RANGE), ("topk", {3: -1}, RANGE), ("topk", {3: (1 << 30) + 1}, RANGE), ("balance", {4: (1 << 30) + 1}, RANGE),
    ("linear", {2: (1 << 30) + 1}, RANGE), ("linear", {2: 1 << 30, 6: 1 << 20, 10: 1 << 20}, RANGE), ("quantize", {6: (1 << 30) + 1, 3: (1 << 30) + 1}, RANGE),
    ("combine", {6: (1 << 30) + 1}, RANGE), ("topk", {4: 0}, RANGE),
    ("topk", {4: 513, 2: 513}, RANGE), ("topk", {5: 0}, RANGE), ("topk", {5: 9}, RANGE), ("topk", {5: 17, 4: 64, 2: 64}, RANGE), ("topk", {6: 2}, INVALID),
    ("topk", {9: None}, INVALID), ("topk", {10: None}, INVALID),
    ("topk_grad", {0: None}, INVALID), ("topk_grad", {12: 7}, RANGE), ("topk_grad", {11: None}, INVALID), ("topk_grad", {8: None}, INVALID),
    ("order", {0: None}, INVALID), ("order", {1: -1}, RANGE), ("order", {1: (1 << 24) + 1}, RANGE), ("order", {2: 0}, RANGE), ("order", {2: 513}, RANGE),
    ("order", {3: None}, INVALID), ("order", {1: 16385}, INVALID), ("order", {1: 16385, 6: P, 7: 8}, INVALID), ("order", {1: 16385, 6: P + 4, 7: 1 << 20}, INVALID),
    ("balance", {0: None}, INVALID), ("balance", {3: None}, INVALID), ("balance", {9: 0}, RANGE), ("balance", {9: 65537}, RANGE), ("balance", {9: 2}, INVALID),
    ("balance", {10: None}, INVALID), ("balance", {14: P + 1}, INVALID), ("balance", {6: 9}, RANGE),
    ("balance_grad", {14: 7}, RANGE), ("balance_grad", {10: None}, INVALID), ("balance_grad", {8: P, 9: 0}, RANGE),
    ("quantize", {1: 0}, INVALID), ("quantize", {7: 72}, UNSUPPORTED), ("quantize", {7: 8}, RANGE), ("quantize", {7: 131072, 2: 131072}, RANGE),
    ("quantize", {2: 63}, RANGE), ("quantize", {6: 5}, RANGE), ("quantize", {4: P, 5: 0}, RANGE), ("quantize", {6: -1}, RANGE), ("quantize", {8: P + 8}, INVALID),
    ("quantize", {0: None}, INVALID), ("quantize", {9: None}, INVALID),
    ("linear", {2: -1}, RANGE), ("linear", {3: 8}, RANGE), ("linear", {3: 72}, UNSUPPORTED), ("linear", {3: 131072}, RANGE), ("linear", {6: 0}, RANGE),
    ("linear", {10: 7}, RANGE), ("linear", {9: 5}, INVALID), ("linear", {0: None}, INVALID), ("linear", {0: P + 8}, INVALID), ("linear", {4: P + 4}, INVALID),
    ("linear", {8: None}, INVALID),
    ("grouped", {8: None}, INVALID), ("grouped", {6: 0}, RANGE), ("grouped", {6: 513}, RANGE), ("grouped", {6: 512, 7: 1 << 23, 12: 1 << 23}, RANGE),
    ("combine", {0: None}, INVALID), ("combine", {1: 9}, INVALID), ("combine", {2: 7}, RANGE), ("combine", {7: 0}, RANGE), ("combine", {7: 17}, RANGE),
    ("combine", {8: 0}, RANGE), ("combine", {8: 8388481, 2: 8388481, 10: 8388481}, RANGE), ("combine", {10: 7}, RANGE), ("combine", {5: None}, INVALID),
    ("combine_grad", {1: 3}, INVALID), ("combine_grad", {6: -1}, RANGE), ("combine_grad", {7: 17}, RANGE), ("combine_grad", {8: 0}, RANGE),
    ("combine_grad", {2: 7}, RANGE), ("combine_grad", {10: 7}, RANGE), ("combine_grad", {13: 7}, RANGE), ("combine_grad", {4: None}, INVALID),
    ("combine_grad", {9: None}, INVALID), ("combine_grad", {11: None}, INVALID),
]


@pytest.mark.parametrize("which,change,code", REFUSED, ids=["%s-%d" % (r[0], i) for i, r in enumerate(REFUSED)])
def test_refused_with_a_message(which, change, code):
    lib = mix.load_library()
    args = list(SMALL_NORMAL[which])
    for i, v in change.items():
        args[i] = v
    err = C.create_string_buffer(256)
    assert getattr(lib, FN[which])(*args, None, err, 256) == code
    assert len(err.value) > 4
    assert getattr(lib, FN[which])(*args, None, None, 0) == code          # without a buffer for the message


def test_workspace_sizes():
    lib = mix.load_library()
    assert lib.mix_expert_order_workspace(0, 8) == 0 and lib.mix_expert_order_workspace(16384, 8) == 0
    assert lib.mix_expert_order_workspace(16385, 8) >= 9 * 9 * 4
    assert lib.mix_expert_order_workspace(1 << 24, 512) > 0
    assert lib.mix_expert_order_workspace((1 << 24) + 1, 8) < 0 and lib.mix_expert_order_workspace(5, 0) < 0
    assert lib.mix_router_balance_workspace(-1, 8, 1) == RANGE and lib.mix_router_balance_workspace(4, 513, 1) == RANGE
    assert lib.mix_router_balance_workspace(4, 8, 0) == RANGE


def test_tensors_of_the_host_are_refused():
    x, i = torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32)
    for call in (lambda: mix.router_topk(x, 2), lambda: mix.router_topk_grad(x, i, x, x), lambda: mix.expert_order(i, 8), lambda: mix.router_balance(x, i),
                 lambda: mix.router_balance_grad(x, i, i, i, x), lambda: mix.quantize_rows(x.bfloat16()),
                 lambda: mix.linear_int(x.char(), x, x.char(), x), lambda: mix.linear_int_grouped(x.char(), x, x.char(), x, i),
                 lambda: mix.expert_combine(x, x, i), lambda: mix.expert_combine_grad(x, x, x, i)):
        with pytest.raises(ValueError):
            call()
