"""Norm and losses claim no more alignment of memory than callers promise: 16 bytes, and 4 within rows of logits (CPU only)."""
import pytest

from tests.test_operand_alignment import test_no_access_claims_more_than_the_contract as claims_no_more


@pytest.mark.parametrize("source", ["norm.hip", "balance.hip"])
def test_no_access_claims_more_than_the_contract(source, tmp_path):
    claims_no_more(source, tmp_path)
