"""Layer norm's row shapes: of two kernels for one kind of rows that hold equally many elements, one could never be launched."""
import collections
import re

from test_operator_resources import kernels, pytestmark  # noqa: F401


def test_no_two_shapes_hold_rows_of_one_length(kernels):  # noqa: F811
    held = collections.defaultdict(list)
    for name in kernels:
        m = re.search(r"k_layer_norm_(forward|backward)I(.+?)Li(\d+)ELi(\d+)ELi(\d+)ELb(\d)E", name)
        if m:
            way, types, team, elements, vector, flag = m.groups()
            held[way, types, flag, vector == "1"].append(int(team) * int(elements))
    assert len(held) == 2 * 5 * 2 * 2                        # passes, types, residual or sums, rows shorter than a vector
    assert not {k: v for k, v in held.items() if len(v) != len(set(v))}
