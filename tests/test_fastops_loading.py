"""The hook's calls need neither torch's C++ libraries nor the module that is linked to them."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code):
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_the_library_loads_without_the_module_of_the_calls_behind_the_router():
    _run("""
import sys
sys.modules["paper_2607_22595_b200._fastops"] = None         # importing it raises, as it does with another torch
import torch, paper_2607_22595_b200 as mix
lib = mix.load_library()
assert lib.mix_apply(None, None, 0, None, None) == -1 and mix.binding._fast is not None
try:
    mix.router_topk(torch.zeros((4, 8)), 2)
except RuntimeError as e:
    assert "_fastops" in str(e) and torch.__version__.split("+")[0] in str(e)
else:
    raise AssertionError("no error")
""")


def test_the_module_is_loaded_by_the_first_call_behind_the_router():
    _run("""
import sys
import torch, paper_2607_22595_b200 as mix
mix.load_library()
assert "paper_2607_22595_b200._fastops" not in sys.modules
try:
    mix.router_topk(torch.zeros((4, 8)), 2)
except ValueError:
    pass
assert "paper_2607_22595_b200._fastops" in sys.modules
""")


def test_a_module_built_for_another_torch_is_not_used():
    _run("""
import torch, paper_2607_22595_b200 as mix
torch.__version__ = "1.2.3+cu1"
try:
    mix.router_topk(torch.zeros((4, 8)), 2)
except RuntimeError as e:
    assert "1.2.3" in str(e) and "build()" in str(e)
else:
    raise AssertionError("no error")
""")
