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


@pytest.mark.parametrize("rule", [stepq.STEPQ_RULE_DECAY, stepq.STEPQ_RULE_DELTA])
@pytest.mark.parametrize("heads", [8, 16, 32, 64, 96])
def test_one_more_chunk_does_not_change_how_a_long_sequence_is_cut(heads, rule):
    """The number of segments follows the length and the heads without a jump, but for the whole chunks a segment
    takes: of 200 chunks in 32 segments at most, 7 or more each, one more is a seventh at most."""
    sizes = [stepq.stepq_prompt_workspace(64 * c, 1, heads, heads, 128, 128, rule) for c in range(200, 600)]
    assert all(a <= 1.25 * b and b <= 1.25 * a for a, b in zip(sizes, sizes[1:]))
