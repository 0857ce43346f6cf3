"""Calls of the shared contexts and of the cache with accumulated weights that lie at the edge of what they take."""
import pytest
import torch

from test_gpu_mass import DT, INF, _i32, _rnd, _sh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("partial", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_no_contexts(dtype, partial):
    """A batch without contexts: all rows belong to nobody."""
    sh, dt, tokens = _sh(), DT[dtype], 6
    q, k = _rnd(1)(tokens, 4, 64, dtype=dt), torch.empty(0, 2, 5, 64, dtype=dt, device="cuda")
    odt = torch.float32 if partial else dt
    for at in (0, 3, tokens):
        for lengths in (None, _i32([])):
            # (whoever asks for memory of these sizes next gets it as it is here)
            left = [torch.full((tokens, 4, 64), 7.0, dtype=odt, device="cuda"), torch.full((tokens, 4), 7.0, device="cuda")]
            del left
            out, lse = sh.context_attention(q, k, k, _i32([at]), lengths, partial=partial)
            assert out.dtype is odt and (out == 0).all() and (lse == -INF).all()
    out, lse = torch.full((tokens, 4, 64), 7.0, dtype=odt, device="cuda"), torch.full((tokens, 4), 7.0, device="cuda")
    sh.context_attention(q, k, k, _i32([2]), partial=partial, out=out, lse=lse)
    assert (out == 7).all() and (lse == 7).all()
