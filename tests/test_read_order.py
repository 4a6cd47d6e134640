"""The loop whose waits count a wave's reads on their way (tile_product_made) pins the order in which it asks, read from the
source: with the two operands' reads free to change places, a count could be met while the buffer that is multiplied next is
still on its way."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2410_22697_amd", "csrc", "tile_product.hpp")


def test_the_asks_of_a_counted_step_stay_in_order():
    with open(SOURCE) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    body = re.search(r"auto step_between = \[&\]\(auto now, auto next\) \{(.*?)\n  \};", text, re.S).group(1)
    calls = [c for c in re.findall(r"tile_arrived<\w+>|tile_barrier|tile_in_order|put|first\.direct|second\.template whole|multiply", body)]
    assert calls == ["tile_arrived<kLeft>", "tile_barrier", "tile_arrived<kLeftPut>", "put", "first.direct", "tile_in_order", "second.template whole",
                     "multiply"]
    order = re.search(r"void tile_in_order\(\) \{(.*?)\n\}", text, re.S).group(1)
    assert 'asm volatile("" ::: "memory")' in order and "__builtin_amdgcn_sched_barrier(" in order
