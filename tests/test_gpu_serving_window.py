"""A long conversation in the serving example: the pages in use stay within what the window needs,
and the logits are what they are with every page kept."""
import pytest
import torch

from tests.test_gpu_hybrid_serving import ex  # noqa: F401

pytestmark = pytest.mark.gpu


def test_pages_stay_within_the_window(ex):  # noqa: F811
    model = ex.HybridModel(window=40)
    g = torch.Generator().manual_seed(3)
    a, b = (torch.randint(0, 211, (n,), generator=g).tolist() for n in (75, 9))
    ids = torch.randint(0, 211, (300, 3), generator=g).cuda()
    # a window of 40 lies in at most 4 pages of 16, the next token's page among them
    small = ex.Server(model, S=3, num_pages=14, max_tokens=400)
    large = ex.Server(model, S=3, num_pages=90, max_tokens=400)
    large._release = lambda: None
    got = []
    for server in (small, large):
        logits = [server.prefill([a, b, []])]
        server.select([0, 1, 0])
        for step in range(300):
            logits.append(server.decode(ids[step]))
            if server is small:
                assert int((server.refs > 0).sum()) <= 12
                held = torch.bincount(server.table[server.table >= 0].long(), minlength=14)
                assert torch.equal(held.to(torch.int32), server.refs)
            if step == 200:
                server.select([2, 1, 1])
                server.compact()
        got.append(torch.stack(logits))
    assert small.lens.tolist() == large.lens.tolist() == [375, 309, 309]
    assert torch.equal(*got)
