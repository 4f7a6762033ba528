"""Refusals of the operators for models whose layers the caller runs that the host makes before anything is enqueued (no GPU)."""

import pytest

from paper_2504_02921_amd import binding as hb
from test_operators_host import FAKE, attend, pool_handle, tables


def test_attention_does_not_write_over_what_it_reads():
    pool = pool_handle()
    apart = dict(q=FAKE + (1 << 20), k=FAKE + (2 << 20), v=FAKE + (3 << 20), out=FAKE + (4 << 20), lse=FAKE + (5 << 20), slopes=FAKE + (6 << 20), prefix_lens=FAKE + (7 << 20))
    for n_pairs in (1, 3):
        t = tables(pool, n_pairs=n_pairs)
        for name in ("q", "k", "v", "lse"):
            assert attend(pool, t, **dict(apart, out=apart[name])) == hb.HR_ERR_INVALID_ARG, name
        for name in ("q", "k", "v", "slopes", "prefix_lens"):
            assert attend(pool, t, **dict(apart, lse=apart[name])) == hb.HR_ERR_INVALID_ARG, name


def test_rotary_sizes_that_would_wrap_around_are_refused():
    """A rotary_dim of 64 - 2^32 would be taken for 64, with room for no frequency."""
    for change in (dict(head_dim=(1 << 32) + 64), dict(rotary_dim=(1 << 32) + 64), dict(head_dim=-64), dict(rotary_dim=-2), dict(rotary_dim=64 - (1 << 32))):
        with pytest.raises(hb.HrError):
            hb.Rope(**{**dict(head_dim=64), **change})
    with pytest.raises(hb.HrError):
        hb.Rope(64, rotary_dim=(1 << 32) + 64, freqs=[0.5] * 32)
