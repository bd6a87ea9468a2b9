"""The example that serves with quantized caches, one selected page a token: the last one, which always is."""
import pytest
import torch

from test_gpu_cache_together import example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P", [40, 150])
def test_one_selected_page(P):
    m = example()
    outs = {}
    for select in (0, 1):
        stack = m.Stack(kinds=("delta", "attention", "decay"), width=128, v_heads=4, qk_heads=2, d=64, q_heads=8, kv_heads=2,
                        head_dim=64, dtype=torch.float32)
        g = torch.Generator().manual_seed(3)
        draw = lambda n: torch.randn((n, stack.width), generator=g)
        prefix, prompts, more = draw(P), [draw(n) for n in (1, 70, 13)], [draw(3) for _ in range(3)]
        server = m.Server(stack, prefix.cuda(), 3, 80, page=16, quantized=False, cache_bits=8, select=select)
        outs[select] = [server.admit([p.cuda() for p in prompts])] + [server.step(x.cuda()) for x in more]
        if select:
            last = (P + server.lengths - 1) // 16
            assert torch.equal(server.selected, last.to(torch.int32)[:, None, None].expand(3, 2, 1))
    assert torch.equal(outs[1][0], outs[0][0])                   # prompts read all pages
    assert torch.isfinite(torch.stack(outs[1])).all()
    assert not torch.equal(outs[1][3], outs[0][3])
