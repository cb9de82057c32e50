"""Workspace sizes of the paged attention call (CPU)."""

import pytest

from paper_2509_00195_amd import make_desc, tts_paged_decode_workspace_size

SEQS = [1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 85, 86, 127, 128, 129, 255, 256, 300, 511, 512, 513, 1000]
LENS = [1, 16, 256, 257, 511, 512, 513, 1000, 1024, 4096, 5000, 120000]


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp8", "mx4"])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (12, 2, 128), (15, 5, 64), (34, 2, 64), (600, 600, 64), (1, 1, 64)])
def test_a_size_serves_every_smaller_batch(kind, hq, hkv, d):
    desc = make_desc(hq, hkv, d, 16, "f32" if kind == "f32" else "bf16", kind)
    size = {(n, m): tts_paged_decode_workspace_size(desc, n, m) for n in SEQS for m in LENS}
    for n, n1 in zip(SEQS, SEQS[1:]):
        for m, m1 in zip(LENS, LENS[1:]):
            assert size[n, m] <= size[n1, m] and size[n, m] <= size[n, m1], (n, m)


def test_a_4_bit_batch_that_is_not_split_itself():
    desc = make_desc(28, 4, 128, 16, "bf16", "mx4")
    assert tts_paged_decode_workspace_size(desc, 128, 4096) >= tts_paged_decode_workspace_size(desc, 127, 4096) > 0
