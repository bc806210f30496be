"""The serving example: prompts, single tokens, forks, ended rows and a compacted
cache give what a prompt of the same tokens gives."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location(
        "hybrid_serving", os.path.join(ROOT, "examples", "hybrid_serving.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def close(a, b):
    """Two routes through the stack in bfloat16: the same values up to roundings of 2^-8 that pass
    through four layers (each an average of many values, rounded a few times), against the
    logits' size of about 1."""
    return ((a.float() - b.float()).abs().max() <= 16 * 2.0 ** -8 * b.float().abs().max())


def test_decoding_equals_a_prompt(ex):
    g = torch.Generator().manual_seed(1)
    model = ex.HybridModel()
    rows = [torch.randint(0, 211, (n,), generator=g).tolist() for n in (150, 3, 97, 40)]
    server = ex.Server(model, S=4)
    server.prefill([r[:-8] if len(r) > 8 else r[:1] for r in rows])
    done = [len(r) - 8 if len(r) > 8 else 1 for r in rows]
    for step in range(8):
        ids = torch.tensor([r[min(done[i] + step, len(r) - 1)] for i, r in enumerate(rows)]).cuda()
        logits = server.decode(ids)
    whole = ex.Server(model, S=4)
    want = whole.prefill(rows)
    for i in (0, 2, 3):
        assert close(logits[i], want[i]), i


def test_forks_ends_and_compaction(ex):
    g = torch.Generator().manual_seed(2)
    model = ex.HybridModel()
    a, b = (torch.randint(0, 211, (n,), generator=g).tolist() for n in (61, 20))
    tails = torch.randint(0, 211, (3, 12), generator=g)
    server = ex.Server(model, S=4, num_pages=40)
    server.prefill([a, b, [], []])
    assert not server.select([0, 0, 1, 0]).any()
    for step in range(12):
        ids = torch.stack([tails[0, step], tails[1, step], tails[0, step], tails[2, step]]).cuda()
        logits = server.decode(ids)
        if step == 5:  # row 3 ends, 2 and 1 change places, the pages are packed
            server.select([0, 2, 1, -1])
            used = server.compact()
            assert (server.refs[:used] > 0).all() and not server.refs[used:].any()
            tails = torch.stack([tails[0], tails[0], tails[1]])
            # from here on row 1 is b's, row 2 the fork of a with the old second tail
            order = [0, 0, 2, 2]
            for s in range(6, 12):
                ids = torch.stack([tails[k, s] for k in order]).cuda()
                logits = server.decode(ids)
            break
    whole = ex.Server(model, S=4)
    t0, t1 = tails[0].tolist(), tails[2].tolist()
    want = whole.prefill([a + t0, b + t0, a + t1, []])
    for i in range(3):
        assert close(logits[i], want[i]), i


def test_main_runs(ex, capsys):
    ex.main()
    out = capsys.readouterr().out
    assert "lengths [94, 94, 25, 57, 174, 174, 174, 24]" in out
