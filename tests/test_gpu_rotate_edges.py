"""Rotary positions at the ends of their arguments' ranges (definition and tolerance: test_gpu_rotate.py)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from chunk_ref import D  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402
from test_gpu_rotate import DEV, L  # noqa: E402


def test_a_single_row_of_any_stride():
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.standard_normal(7 * D).astype(np.float16)).to(DEV)
    pos = torch.tensor([12345], dtype=torch.int32, device=DEV)
    freq, _ = dk.rope_frequencies(128)
    q = x[:4 * D].as_strided((1, 4, D), (3, D, 1))
    out, _ = dk.rotate(L, pos, freq.to(DEV), q)
    want, _ = dk.rotate(L, pos, freq.to(DEV), x[:4 * D].view(1, 4, D))
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_more_rows_than_a_launch_has_waves():
    """2^26 rows and a few, of one head: the last ones (and some of each part of the way) are turned as any others."""
    rows = (1 << 26) + 5
    x = torch.empty((rows, 1, D), dtype=torch.float16, device=DEV)
    at = torch.tensor([0, 1, 1 << 24, (1 << 24) + 3, (1 << 25) - 1, (1 << 26) - 1, 1 << 26, rows - 1], device=DEV)
    x[at] = torch.randn((len(at), 1, D), device=DEV).half()
    pos = torch.arange(rows, dtype=torch.int32, device=DEV)
    freq = dk.rope_frequencies(128)[0].to(DEV)
    want, _ = dk.rotate(L, pos[at], freq, x[at])
    print("case: 2^26 rows", flush=True)
    dk.rotate(L, pos, freq, x, q_out=x)
    torch.cuda.synchronize()
    assert torch.equal(x[at], want)
