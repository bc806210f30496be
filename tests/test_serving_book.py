"""The book-keeping of the serving example, without a GPU: the page call is a stand-in."""
import importlib.util
import os

import pytest
import torch

from paper_2412_06464_amd import gdn, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def server():
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    spec = importlib.util.spec_from_file_location(
        "hybrid_serving", os.path.join(ROOT, "examples", "hybrid_serving.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod.Server(mod.HybridModel(device="cpu", window=40), S=3, page_size=16, num_pages=30,
                      max_tokens=160)


@pytest.mark.parametrize("call", [lambda s: s.decode(torch.zeros(3, dtype=torch.long)),
                                  lambda s: s.prefill([[1, 2], [], [3]])])
def test_no_pages_left(server, monkeypatch, call):
    """The call ends with an error that optimised code keeps, and no row has grown."""
    def extend(table, lens, refs, add, page_size):
        return dict(table=table + 1, lens=lens + add, refs=refs + 1,
                    short=torch.tensor([0, 2, 0], dtype=torch.int32))
    monkeypatch.setattr(paged, "gdn_pages_extend", extend)
    before = [x.clone() for x in (server.table, server.lens, server.refs)]
    with pytest.raises(RuntimeError, match=r"no pages left for rows \[1\]"):
        call(server)
    assert all(torch.equal(x, y) for x, y in zip(before, (server.table, server.lens, server.refs)))


def test_pages_behind_the_window_are_released(server):
    """A page goes when its last token is one that no row's next token sees; shared ones when
    their last holder lets go; holes stay holes."""
    P = server.page
    server.table[0, :4] = torch.tensor([7, 3, 9, 5])
    server.table[1, :4] = torch.tensor([7, 3, -1, 2])
    server.table[2, :2] = torch.tensor([7, 1])
    server.lens = torch.tensor([4 * P, 4 * P - 9, P + 1], dtype=torch.int32)
    server.refs[torch.tensor([7, 3, 9, 5, 2, 1])] = torch.tensor([3, 2, 1, 1, 1, 1],
                                                                 dtype=torch.int32)
    # the next tokens, at 64, 55 and 17, see from 25, 16 and 0 on
    server._release()
    assert server.table[:, :5].tolist() == [[-1, 3, 9, 5, -1], [-1, 3, -1, 2, -1], [7, 1, -1, -1, -1]]
    assert [server.refs[p].item() for p in (7, 3, 9, 5, 2, 1)] == [1, 2, 1, 1, 1, 1]
    server.lens[:2] += torch.tensor([7, 16], dtype=torch.int32)  # see from 32 on
    server._release()
    assert server.table[:, :5].tolist() == [[-1, -1, 9, 5, -1], [-1, -1, -1, 2, -1],
                                            [7, 1, -1, -1, -1]]
    assert [server.refs[p].item() for p in (7, 3, 9, 5, 2, 1)] == [1, 0, 1, 1, 1, 1]
    assert server.refs.dtype is torch.int32 and server.table.dtype is torch.int32
