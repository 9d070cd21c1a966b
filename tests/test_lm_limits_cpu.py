"""Calls of the language-model operators that are more than a launch takes: refused before anything is enqueued, here
without a GPU."""
import pytest

from paper_2505_05086_amd import binding as B

P = 0x10000          # non-null, 256-aligned, never dereferenced by validation
UNSUPPORTED = 2


@pytest.mark.parametrize("out_dtype", [B.ASI_F32, B.ASI_BF16])
@pytest.mark.parametrize("tokens,dim", [(1024, 1 << 24), (1 << 20, 1 << 23), (1 << 29, 1 << 24), (1024, (1 << 24) - 1)])
def test_embedding_gradients_of_more_workgroups_than_a_launch_has(tokens, dim, out_dtype):
    desc = B.EmbeddingDesc(tokens, 100, dim, dim, dim, -1, B.ASI_F32, out_dtype, 1.0, 0)
    assert B.lib().asi_embedding_grad(desc, P, P, P, 0, P, 1 << 62, None) == UNSUPPORTED


def test_the_version_tells_libraries_with_these_entry_points_apart():
    assert B.asi_version() >= 1003
