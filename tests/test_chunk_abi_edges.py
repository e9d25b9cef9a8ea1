"""Sizes and refusals of the chunk operators and rotary positions at the ends of their ranges (CPU only; no call
here reaches a kernel)."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def dk():
    from paper_2412_03131_amd import diffkv
    if not os.path.exists(diffkv.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    diffkv.lib()
    return diffkv


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (32, 32), (8, 1), (5, 5), (64, 8), (28, 4), (1024, 1024), (1200, 1200)])
def test_a_workspace_for_more_sequences_serves_fewer(dk, Hq, Hkv):
    """The size never falls as the batch grows, past the batch from which tables are not split too (1024 tables)."""
    L = dk.layout(max_seq_len=4096)
    border = -(-1024 // Hkv)
    seqs = sorted({s for s in (*range(1, 70), 127, 128, 129, border - 1, border, border + 1, 4 * border) if s > 0})
    for rows in (1, 2, 31, 32, 64, 65, 127, 128, 300, 1024, 8192, 70000):
        need = [dk.workspace_size(dk.OP_CHUNK_ATTENTION, L, s, Hq, Hkv, rows) for s in seqs]
        assert need == sorted(need), rows
        need = [dk.workspace_size(dk.OP_CHUNK_SIGNIFICANCE, L, s, Hq, Hkv, rows) for s in seqs]
        assert need == sorted(need), rows


def test_scales_beyond_the_range_of_scores(dk):
    """Scores as large as the kernels' running maximum can start below: refused with their scale."""
    from test_chunk_abi import attention, significance
    for scale in (65537.0, 1e8, 1e30):
        assert attention(dk, scale=scale) == dk.E_INVAL
        assert significance(dk, scale=scale) == dk.E_INVAL
    assert attention(dk, scale=65536.0) == dk.E_WORKSPACE  # (the next check: none is given)


def test_binding_refuses_host_tensors(dk):
    """What diffkv_rope_frequencies gives lies on the host; a kernel that took such an address would fault."""
    L = dk.layout(max_seq_len=256)
    q, kv = torch.zeros((3, 8, 128), dtype=torch.float16), torch.zeros((3, 2, 128), dtype=torch.float16)
    freq, _ = dk.rope_frequencies(128)
    with pytest.raises(ValueError, match="GPU"):
        dk.rotate(L, torch.zeros(3, dtype=torch.int32), freq, q, kv)
    cache = dk.Cache(L, 16, 1, 2, device="cpu")
    nl, ws = torch.tensor([3], dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        dk.chunk_attention(cache, nl, q, kv, kv, 0.1, max_new=3, ws=ws)
    with pytest.raises(ValueError, match="GPU"):
        dk.chunk_significance(cache, nl, q, kv, 0.1, torch.zeros((3, 8)), max_new=3, ws=ws)


@pytest.mark.parametrize("stride", [-1, 0, 3, 1 << 40])
def test_a_single_row_has_any_stride(dk, stride):
    from test_chunk_abi import attention, significance
    strides = dict(total=1, max_new=1, qs=stride, ks=stride)
    assert attention(dk, vs=stride, **strides) == dk.E_WORKSPACE  # (past the rows' checks: none is given)
    assert significance(dk, **strides) == dk.E_WORKSPACE


def test_more_tables_than_a_launch_can_take(dk):
    """A launch has less than 2^32 threads, and gives no error beyond."""
    from test_chunk_abi import attention, significance
    for seqs, status in ((1 << 21, dk.E_WORKSPACE), ((1 << 21) + 1, dk.E_UNSUPPORTED), (1 << 28, dk.E_UNSUPPORTED)):
        assert attention(dk, seqs=seqs) == status
        assert significance(dk, seqs=seqs) == status


def test_workspace_of_more_rows_than_a_call_takes(dk):
    """Row counts that the calls refuse have no size either (their products would not fit 64 bits)."""
    L = dk.layout(max_seq_len=256)
    for op in (dk.OP_CHUNK_ATTENTION, dk.OP_CHUNK_SIGNIFICANCE):
        for rows in ((1 << 29), 1 << 60):
            with pytest.raises(dk.DiffKVError) as e:
                dk.workspace_size(op, L, 4, 32, 8, rows)
            assert e.value.code == dk.E_INVAL
        assert dk.workspace_size(op, L, 4, 32, 8, (1 << 29) - 1) > 0
