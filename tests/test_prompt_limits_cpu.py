"""Limits of the operators of a prompt's pass: what the header names is taken, what a launch cannot hold is refused, before any HIP
call."""
from __future__ import annotations

import re

import pytest

from test_prompt_cpu import CHUNK, attend, pr  # noqa: F401

FAKE = 0x100000  # never read: every call fails its checks first
LARGEST = (1 << 24) - 4096  # (rows * group / 128 + seqs) * kv_heads


def config(pr, **kw):  # noqa: F811
    return pr.argus_chunk_config(*{**CHUNK, "columns": 1, **kw}.values())


@pytest.mark.parametrize("columns,window", [(1, 0), (1 << 20, 0), (1 << 20, 500)])
@pytest.mark.parametrize("head_dim", [64, 128, 256])
@pytest.mark.parametrize("rows,group,seqs,kv_heads", [
    (100, 4, (1 << 20) - 256 - 4, 16), (4192280 * 32, 4, 1000, 4), (4096 * 32 - 1024 - 128, 128, 1, 128),
    (0, 1, 1 << 20, 15), (1863680, 1, 1820, 1024), (16379 * 128, 1, 1, 1024), (2047 * 16, 1, 16125 - 256, 1024)])
def test_largest_batches_are_taken(pr, rows, group, seqs, kv_heads, head_dim, columns, window):  # noqa: F811
    assert (rows * group // 128 + seqs) * kv_heads <= LARGEST and rows * group < 1 << 30
    kw = dict(rows=rows, group=group, seqs=seqs, kv_heads=kv_heads, head_dim=head_dim, columns=columns, window=window)
    assert pr.argus_prompt_attend_workspace_bytes(config(pr, **kw)) < 1 << 40
    # a buffer of no records: refused with how many there would be, two of a wave of 64 threads, of all launches (up to 16
    # waves are the plan's, and 768 x 8 blocks of four join)
    from paper_2609_12299_amd import argus_decode_last_error
    rc = attend(pr, markers=pr.argus_markers(FAKE, 0, 0, 0, 0), io_kw=dict(table_stride=columns), **kw)
    if rows:
        assert rc == -4
        records = int(re.search(r"(\d+) marker records", argus_decode_last_error()).group(1))
        assert (records // 2 - (16 + 768 * 8 * 4 if columns > 1 else 0)) * 64 < 1 << 32


@pytest.mark.parametrize("columns", [1, 1 << 20])
@pytest.mark.parametrize("rows,group,seqs,kv_heads", [
    (100, 4, 1 << 20, 16), (1 << 21, 1, 1, 1024), (1 << 23, 64, 1, 16), (1 << 20, 256, 1 << 20, 8)])
def test_more_than_a_launch_holds_is_refused(pr, rows, group, seqs, kv_heads, columns):  # noqa: F811
    for head_dim in (64, 128, 256):
        kw = dict(rows=rows, group=group, seqs=seqs, kv_heads=kv_heads, head_dim=head_dim, columns=columns)
        assert attend(pr, **kw) == -4
        assert pr.argus_prompt_attend_workspace_bytes(config(pr, **kw)) == (1 << 64) - 1


def test_starts_have_one_dimension(monkeypatch):
    import torch

    from paper_2609_12299_amd import ArgusError, prompt, rotate_tokens
    prompt._t()
    monkeypatch.setattr(prompt, "_elsewhere", lambda stream, dev: False)
    q, f = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.ones(32, dtype=torch.float64)
    for starts in (torch.zeros((), dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32)):
        with pytest.raises(ArgusError, match="starts"):
            rotate_tokens(q, None, None, None, None, None, starts, f, torch.tensor([0, 3]).int())
