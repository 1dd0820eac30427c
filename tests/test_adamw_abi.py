"""What a step of AdamW refuses and accepts at the C ABI, on the CPU."""
import pytest

import paper_2201_07598_amd as okt
from paper_2201_07598_amd import binding
from test_operators_abi import INVALID, OK
from test_training_abi import AT


@pytest.mark.parametrize("lr", [float("nan"), float("inf"), -float("inf"), 1e300])
def test_a_rate_on_the_device_is_the_only_one_looked_at(lr):
    def step(d_lr, chunks=0):                    # no chunks: accepted, and nothing is launched
        op = binding._ADAMW.pack(1, chunks, 0, 0, lr, 0.9, 0.999, 1e-8, AT[1], d_lr, 0, 0, 0)
        return okt.load_library().okt_adamw_step(op, AT[0], None)

    assert step(AT[2]) == OK
    assert step(AT[2] + 2) == INVALID and step(0) == INVALID and step(0, 1) == INVALID
