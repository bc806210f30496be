"""The cache's list of sequences to leave alone, as far as the host checks it."""
from tests.test_paged_abi import ALIGN, FAKE, attn, cache, lib, ref, rows, tokens  # noqa: F401


def test_alignment_of_skip(lib):  # noqa: F811
    t, r, a = tokens(), rows(), attn()
    for kw, code in ((dict(skip=FAKE + 2), ALIGN),):
        c = cache(**kw)
        assert lib.gdn_cache_append(ref(t), None, ref(r), ref(r), ref(r), ref(c), ref(r),
                                    None) == code
        assert lib.gdn_cache_attn(ref(t), ref(a), ref(r), ref(c), ref(r), None, None, 0,
                                  None) == code
