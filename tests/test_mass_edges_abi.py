"""Argument checks of the shared contexts at their edges (no device call is made: every call below is refused, or has nothing to do)."""
import pytest

from test_mass_abi import FAKE, _args, _calls, _sh


@pytest.mark.parametrize("change", [dict(out=None), dict(out__data=FAKE + 8), dict(out__token_stride=128), dict(lse=None), dict(lse=FAKE + 2), dict(q=None),
                                    dict(starts=None), dict(starts=FAKE + 2), dict(lengths=FAKE + 1)])
def test_rows_that_are_cleared_are_looked_at_without_contexts_too(change):
    sh = _sh()
    x = _args(sh)
    x["n"], x["clear"], x["cache"] = 0, 1, None
    for name, value in change.items():
        if "__" in name:
            setattr(x[name.split("__")[0]], name.split("__")[1], value)
        else:
            x[name] = value
    assert _calls(sh, x)["context"]() == sh.SH_EINVAL
    if change == dict(starts=None):
        return
    x["clear"] = 0                                                        # nothing is written then
    assert _calls(sh, x)["context"]() == sh.SH_OK


def test_no_tokens_and_no_contexts():
    sh = _sh()
    x = _args(sh)
    x["n"] = x["tokens"] = 0
    for clear in (0, 1):
        x["clear"] = clear
        assert _calls(sh, x)["context"]() == sh.SH_OK
