"""Outputs of the linear-attention block's entry points over their small inputs:
slopes, lengths and slots, which later workgroups and launches read again.
Refused before any GPU work, like what test_linear_block_args has."""
import pytest

from paper_2607_12358_amd import _lib as L
from test_linear_block_args import BAD, G, _attend, _step, lib  # noqa: F401  (lib: fixture)

O_BYTES, STATES = 2 * 3 * 100 * 64 * 2, 2 * 3 * 64 * 64 * 4   # _attend's sizes
LONG = dict(n=1, heads=2, L=40000, ld=40000, d=128)           # takes a workspace
O_LAST, POOL = 3 * 128 * 2, 9 * 2 * 64 * 64 * 4               # _step's: o's last row, the pool


@pytest.mark.parametrize("small,size", [("slopes", 3 * 4), ("lengths", 2 * 4)])
def test_prompts(lib, small, size):  # noqa: F811
    for at in (5 * G, 5 * G + O_BYTES - 4, 5 * G - size + 4):
        assert _attend(lib, **{small: at}) == BAD and small in L.last_error()
    for at in (7 * G, 7 * G + STATES - 4, 7 * G - size + 4):
        assert _attend(lib, sout=7 * G, **{small: at}) == BAD and small in L.last_error()
        assert _attend(lib, sin=7 * G, sout=7 * G, **{small: at}) == BAD and small in L.last_error()


def test_workspace(lib):  # noqa: F811
    need = lib.acid_linear_attention_workspace_needed(L.ACID_BF16, 1, 2, 40000, 128, 0)
    assert need > 0
    for small in ("slopes", "lengths"):
        for at in (6 * G, 6 * G + need - 4):
            assert _attend(lib, bytes=need, **LONG, **{small: at}) == BAD
            assert "workspace" in L.last_error()


@pytest.mark.parametrize("small,size", [("slopes", 2 * 4), ("slots", 4 * 4)])
def test_steps(lib, small, size):  # noqa: F811
    for at in (5 * G, 5 * G + O_LAST, 5 * G + O_LAST + 252, 5 * G - size + 4):
        assert _step(lib, **{small: at}) == BAD and small in L.last_error()
    for out in (4 * G, 7 * G):  # in place and apart
        for at in (out, out + POOL - 4, out - size + 4):
            assert _step(lib, sout=out, **{small: at}) == BAD and small in L.last_error()
