"""What an AdamWPlan refuses about memory that is shared, and what it takes."""
import pytest
import torch

from paper_2506_03077_b200 import binding as B

pytestmark = pytest.mark.gpu


def entry(buf, **at):
    """An entry of 64 elements at the given offsets into one fp32 buffer."""
    return {k: buf[o:o + 64] for k, o in at.items()}


def test_shared_memory():
    buf = torch.zeros(1024, device="cuda")
    first = dict(param=0, grad=64, m=128, v=192)
    second = dict(param=256, grad=320, m=384, v=448)
    B.AdamWPlan([entry(buf, **first), entry(buf, **second)])
    B.AdamWPlan([entry(buf, **first), entry(buf, **(second | dict(grad=64)))])            # a shared gradient is only read
    B.AdamWPlan([entry(buf, **first), {k: buf[:0] for k in first}])
    for bad in (dict(param=128), dict(m=100), dict(v=256), dict(grad=256), dict(grad=0), dict(grad=100), dict(grad=160), dict(grad=448),
                dict(grad=500)):
        with pytest.raises(ValueError, match="overlap"):
            B.AdamWPlan([entry(buf, **first), entry(buf, **(second | bad))])
