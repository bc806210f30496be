"""The kernel of few rows on packed input, and rotary positions element by element, against
64 bits."""
import pytest
import torch

from tests.paged_ref import Case, turn
from tests.test_gpu_paged_batches import check, run
from tests.test_gpu_paged_rows import theta_of

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
HEADS = [(BF, 64, 4, 4), (BF, 64, 16, 1), (BF, 128, 8, 2), (BF, 128, 3, 1), (BF, 256, 6, 2),
         (F32, 64, 4, 2), (F32, 128, 2, 2), (F32, 256, 3, 1)]


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


@pytest.mark.parametrize("dtype,d,Hq,Hk", HEADS)
@pytest.mark.parametrize("rows", [16, 32])
@pytest.mark.parametrize("window", [0, 1, 20])
def test_packed(P, dtype, d, Hq, Hk, rows, window):
    """At most 16, and 17 to 32, rows a sequence: sequences without new tokens, one whose cache
    holds fewer tokens than are new, an empty cache, holes, a cache long enough to be split."""
    most = rows // (Hq // Hk)
    new = [most, 0, 1, most, 0, (most + 1) // 2, 1]
    kv = [most + 40, 0, 1, most // 2, 33, 2500, 0]
    c = Case(new, kv, Hq, Hk, d, 32, dtype, window, holes={(0, 1), (5, 70)}, seed=d + rows)
    print("[gpu-case] few", dtype, d, Hq, Hk, rows, window, flush=True)
    check(c, *run(P, c))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_packed_not_causal(P, dtype):
    c = Case([3, 0, 2, 1], [40, 9, 700, 1], 8, 2, 128, 16, dtype, causal=False, seed=6)
    check(c, *run(P, c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["halves", "interleaved"])
@pytest.mark.parametrize("d,rot,scaling", [(64, 64, "none"), (128, 126, "parts"), (256, 40, "base")])
def test_rotation_element_by_element(P, dtype, layout, d, rot, scaling):
    """A pair's two products, their sum and the factor's product are off by 2^-24 each; cos and
    sin, the angle's rounding to 32 bits in them, by 2^-22 (bfloat16: the hardware's, 2^-20);
    bfloat16 rounds the result once."""
    g = torch.Generator().manual_seed(d + rot)
    # neighbours of very different size: a bound by the row's largest value would hide the small
    x = torch.randn(2, 23, 3, d, generator=g) * torch.exp2(torch.randint(-12, 3, (2, 23, 3, d),
                                                                          generator=g).float())
    x = x.to(dtype)
    pos = torch.randint(0, 1 << 20, (2, 23), generator=g).to(torch.int32)
    th, scale = theta_of(rot, scaling)
    r = P.gdn_rotary(rot, layout=layout, scaling=scaling, factor=8.0, original=4096)
    i = torch.arange(rot // 2)
    a, b = (i, i + rot // 2) if layout == "halves" else (2 * i, 2 * i + 1)
    size = x.double().abs()
    both = (size[..., a] + size[..., b]) * scale
    trig = 2.0 ** -20 if dtype is BF else 2.0 ** -22
    for f, sign in ((P.gdn_rotary_fwd, 1.0), (P.gdn_rotary_bwd, -1.0)):
        y = f(x.cuda(), None, r, positions=pos.cuda())[0].cpu()
        want = turn(x.flatten(0, 1), pos.flatten(), th, layout, scale, sign).reshape(x.shape)
        off = torch.zeros_like(want)
        off[..., a] = off[..., b] = both * (trig + 4 * 2.0 ** -24)
        if dtype is BF:
            off = off * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
        assert ((y.double() - want).abs() <= off + 1e-30).all()
        assert torch.equal(y[..., rot:], x[..., rot:])
