"""The package loads torch only for what needs it."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_package_loads_torch_for_the_operators_only():
    code = "import sys; import paper_2410_22697_amd as p; assert 'torch' not in sys.modules; p.Massive; p.load; " \
           "assert 'torch' not in sys.modules; assert 'AdamW' in dir(p); p.AdamW; assert 'torch' in sys.modules; " \
           "from paper_2410_22697_amd import RowFormat, linear; assert p.linear is linear; " \
           "import paper_2410_22697_amd.operators as o; assert o.linear is linear and p.operators is o"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)
    code = "import paper_2410_22697_amd as p\ntry:\n    p.nothing\nexcept AttributeError:\n    print('none')"
    assert subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, capture_output=True, text=True).stdout == "none\n"
