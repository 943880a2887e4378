"""Host logic of the packed strategy (paper_2501_08453_amd.memory): which layers, and in which order their outputs are
packed and brought back."""
import itertools

import pytest

from paper_2501_08453_amd import memory as mem


@pytest.mark.parametrize("ratio,selected", [(0.0, 0), (0.2, 2), (0.5, 5), (1.0, 10)])
def test_selected_layers(ratio, selected):
    st = mem.plan(10, ratio, "pack")
    assert st == ["pack"] * selected + ["keep"] * (10 - selected)
    assert mem.device_sets(st) == 10 - selected + (1 if selected else 0) and mem.ring_size(st) == 0


def test_schedules_bring_back_what_was_packed():
    """With any mix of strategies: a packed layer's scratch is packed before another forward overwrites it, and holds its
    outputs again right before its backward."""
    for k in range(1, 6):
        for st in itertools.product(["keep", "recompute", "offload", "pack"], repeat=k):
            st = list(st)
            shared = [i for i, s in enumerate(st) if s in ("recompute", "pack")]
            scratch, packed, done = None, set(), []
            for op in mem.forward_ops(st) + mem.backward_ops(st):
                i = op[1] if len(op) > 1 else None
                if op[0] in ("fwd", "recompute") and i in shared:
                    scratch = i
                elif op[0] == "pack":
                    assert scratch == i and st[i] == "pack"
                    packed.add(i)
                elif op[0] == "unpack":
                    assert i in packed
                    scratch = i
                elif op[0] == "bwd":
                    assert i not in shared or scratch == i
                    done.append(i)
            assert done == list(reversed(range(k))) and packed == {i for i, s in enumerate(st) if s == "pack"}
