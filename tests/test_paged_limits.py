"""CPU checks of the paged calls' largest sizes: what the searches over sequences could not count is refused."""
import pytest

from paper_2503_02356_amd import binding as B
from tests.test_paged_abi import append, paged, refused


@pytest.mark.parametrize("n_seqs", [(1 << 30) + 1, (1 << 31) - 1])
def test_more_sequences_than_the_searches_count_are_refused(n_seqs):
    refused(B.CF_EINVAL, B.cf_attn_paged_fwd, paged(n_seqs=n_seqs))
    refused(B.CF_EINVAL, B.cf_kv_append, append(n_seqs=n_seqs))
    with pytest.raises(B.CfError):
        B.cf_attn_paged_workspace_bytes(paged(n_seqs=n_seqs))


def test_as_many_as_they_count_are_not():
    assert B.cf_attn_paged_workspace_bytes(paged(n_seqs=1 << 30)) == 0
