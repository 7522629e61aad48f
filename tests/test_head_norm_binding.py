"""The binding's head norms built as the C structure that they are, as pools, batches and
rotations may be."""

import pytest

from paper_2609_33536_amd import ekv
from tests.test_serve_bindings import Device, calls  # noqa: F401
from tests.test_serve_host import AT, _pool

torch = pytest.importorskip("torch")
BF, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("norm", [ekv.HeadNorm(AT, AT, 0, 128, 1e-6, 0.0), ekv.HeadNorm(None, AT, 0, 0, 1e-5, 1.0), ekv.HeadNorm(eps=1e-6)])
def test_a_norm_built_by_hand_is_passed_on(calls, norm):  # noqa: F811
    x = lambda h: Device((3, h, 128), BF)  # noqa: E731
    ekv.norm_rope_append(_pool(num_kv_heads=2), ekv.Rope(AT, 128, 0, 1.0), norm, Device((3,), I32), Device((3,), I32), x(8), x(2), x(2), x(8))
    assert [c[0] for c in calls] == ["ekv_norm_rope_append"]
