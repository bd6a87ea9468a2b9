"""How calls around the decode step split their work, as far as the workspace
they ask for tells: host only."""
import pytest
import torch

from paper_2609_38169_amd import stepq


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,D", [(8, 8, 256), (16, 8, 128), (16, 1, 64), (4, 4, 128)])
def test_a_longer_prefix_of_one_request_is_not_cut_in_fewer_parts(hq, hkv, D, act):
    """At most 16 query rows a head read the prefix once in any form: more of it is never a reason for fewer ranges
    (which the form for many rows would take)."""
    sizes = [stepq.stepq_prefix_attention_workspace(1, hq, hkv, D, 1 << i, 1, 16, act) for i in range(4, 21)]
    assert sizes == sorted(sizes), sizes
