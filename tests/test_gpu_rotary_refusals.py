"""rotary_qkv's refusals in Python are ValueErrors: what is missing, and outputs of other axes."""
import numpy as np
import pytest
import torch

from fp8_util import normal
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def test_missing_and_of_other_axes():
    P = need_gpu()
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    q, k, v = (normal((5, 2 * 64), i) for i in range(3))
    ok = dict(q=q, k=k, v=v, positions=torch.zeros((1, 5), dtype=torch.int32, device="cuda"),
              freqs=torch.ones(32, dtype=torch.float64, device="cuda"), sections=(32,), q_out=z(2, 5, 64), k_out=z(2, 5, 64), vt=z(2, 64, 5))
    P.rotary_qkv(**ok)
    for kw, why in ((dict(positions=None), "positions"), (dict(freqs=None), "freqs"), (dict(k_out=z(5, 64)), "k_out"),
                    (dict(k_out=z(64)), "k_out"), (dict(q_out=z(5, 64)), "heads"), (dict(q_out=z(1, 1, 2, 5, 64)), "heads"),
                    (dict(vt=z(64, 5)), "vt"), (dict(q=None, q_out=None, k=None, k_out=None, vt=z(64, 5)), "heads"),
                    (dict(k_out=z(1, 2, 5, 64)), "k_out"), (dict(vt=z(1, 2, 64, 5)), "vt"), (dict(q=z(5, 2, 64)), "rows"),
                    (dict(k=z(5, 2, 64)), "k"), (dict(sections=(32.0,)), "sections"), (dict(sections=(None,)), "sections"),
                    (dict(sections=(1 << 40,)), "freqs"), (dict(sections=32), "sections"), (dict(sections=(1 << 40, -(1 << 40))), "sections"),
                    (dict(q_scale=None), "q_scale"), (dict(eps=None), "eps")):
        with pytest.raises(ValueError, match=why):
            P.rotary_qkv(**{**ok, **kw})
    with pytest.raises(P.AcidError, match="sections"):
        P.rotary_qkv(**{**ok, "sections": (8, -8)})
    for sections in ([32], torch.Size((32,)), np.array([32])):  # any numbers of pairs
        P.rotary_qkv(**{**ok, "sections": sections})
    some = {**ok, "q": None, "q_out": None, "positions": None, "freqs": None}
    with pytest.raises(ValueError, match="positions"):
        P.rotary_qkv(**some)
    P.rotary_qkv(**{**some, "k": None, "k_out": None})  # V alone has no positions
