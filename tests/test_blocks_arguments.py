"""What the calls that fill a cache and read its blocks refuse of tensors that do not go with their structures (no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2404_09336_b200 import ssa


def rows(B=2, heads=2, n_q=3, D=128):
    return torch.zeros(B, heads, n_q, D, dtype=torch.bfloat16)


def cache(B=2, H_kv=2, T=64, D=128):
    return torch.zeros(B, H_kv, T, D, dtype=torch.bfloat16)


def refuses(desc, a, k, v, q=None, q_out=None):
    with pytest.raises(ValueError, match="rows of"):
        ssa.cache_append(desc, a, k, v, None, None, None, q, q_out, stream=0)


def test_rows_of_other_head_counts():
    k, q = rows(), rows(heads=8)
    for bad in (dict(v_new=rows(heads=1)), dict(v_new=rows(heads=8)), dict(q=q, q_out=rows(heads=4)), dict(q=q), dict(q_out=q)):
        with pytest.raises(ValueError, match="heads"):
            ssa.make_append(**{**dict(k_new=k, v_new=k), **bad})


def test_rows_that_the_descriptor_does_not_count():
    q = rows(heads=8)
    desc = ssa.make_desc(q[:, :, 0], cache(), cache(), q[:, :, 0])
    good = ssa.make_append(rows(), rows(), q, q)
    with pytest.raises(ssa.SsaError):                        # (refused by the library: there are no lengths)
        ssa.cache_append(desc, good, rows(), rows(), None, None, None, q, q, stream=0)
    for k, x in ((rows(heads=1), q), (rows(heads=4), q), (rows(D=64), rows(heads=8, D=64)), (rows(), rows(heads=4)), (rows(B=1), rows(B=1, heads=8))):
        refuses(desc, ssa.make_append(k, k, x, x), k, k, x, x)
    k = rows(heads=1)
    refuses(desc, ssa.make_append(k, k), k, k)
    # (queries that are not rotated need not be the descriptor's)
    with pytest.raises(ssa.SsaError):
        ssa.cache_append(desc, ssa.make_append(rows(), rows()), rows(), rows(), None, None, None, stream=0)


def test_rows_of_other_strides_than_the_structure_has():
    q, apart = rows(heads=8), rows().transpose(1, 2).contiguous().transpose(1, 2)
    desc = ssa.make_desc(q[:, :, 0], cache(), cache(), q[:, :, 0])
    good = ssa.make_append(rows(), rows(), q, q)
    refuses(desc, good, apart, rows(), q, q)
    refuses(desc, good, rows(), apart, q, q)
    refuses(desc, good, rows(), rows(), q, rows(heads=4))
    refuses(desc, ssa.make_append(rows(), rows()), rows(), rows(), q, q)
    one = ssa.make_desc(q[:1, :, 0], cache(1, 1), cache(1, 1), q[:1, :, 0])
    k = rows(1, 1)
    with pytest.raises(ssa.SsaError):                        # one request, one head: strides between them do not matter
        ssa.cache_append(one, ssa.make_append(k, k), k.as_strided(k.shape, (7, 5, 128, 1)), k, None, None, None, stream=0)


def chosen(n_q=3):
    q, b = rows(heads=8, n_q=n_q), torch.zeros(2, 2, 2, 2, 128, dtype=torch.bfloat16)
    desc = ssa.make_desc(q[:, :, 0], cache(), cache(), q[:, :, 0])
    return q, b, desc, torch.zeros(2, 2, n_q, 4, dtype=torch.int32), torch.zeros(2, 2, n_q, dtype=torch.int32)


def test_blocks_made_without_the_tensors_that_a_call_takes():
    q, b, desc, index, counts = chosen()
    with pytest.raises(ValueError, match="bounds of other strides"):
        ssa.block_select(desc, ssa.make_blocks(3, 32, 4, q=q), q, b, None, index, counts, stream=0)
    with pytest.raises(ValueError, match="bounds of other strides"):
        ssa.block_bounds(desc, ssa.make_blocks(3, 32, 4, bounds=torch.zeros(2, 3, 2, 2, 128).bfloat16()[:, :2]), None, None, b, stream=0)
    for k, x, out in ((ssa.make_blocks(3, 32, 4, bounds=b), q, q), (ssa.make_blocks(3, 32, 4, q=q, bounds=b), q[:, :, 0], q)):
        with pytest.raises(ValueError, match="q and out"):
            ssa.block_select(desc, k, x, b, None, index, counts, stream=0)
    apart = q.transpose(1, 2).contiguous().transpose(1, 2)
    for k, x, out in ((ssa.make_blocks(3, 32, 4), q, q), (ssa.make_blocks(3, 32, 4, q=q), q, q), (ssa.make_blocks(3, 32, 4, q=q, out=q), q, apart),
                      (ssa.make_blocks(3, 32, 4, q=q, out=q), apart, q)):
        with pytest.raises(ValueError, match="q and out"):
            ssa.attn_blocks(desc, k, x, None, None, None, index, counts, out, stream=0)
    # one token: as the runner calls them
    q, b, desc, index, counts = chosen(1)
    for f in (lambda: ssa.block_select(desc, ssa.make_blocks(1, 32, 4, bounds=b), q[:, :, 0], b, None, index, counts, stream=0),
              lambda: ssa.attn_blocks(desc, ssa.make_blocks(1, 32, 4), q[:, :, 0], None, None, None, index, counts, q[:, :, 0], stream=0)):
        with pytest.raises(ssa.SsaError):
            f()


def test_tokens_that_share_a_row_of_out():
    from test_blocks_abi import attend, desc, good_blocks
    before, k = ssa.launch_count(), good_blocks()
    k.o_stride_t = 0
    assert attend(desc(), k) == ssa.ERR_UNSUPPORTED and ssa.launch_count() == before


@pytest.mark.parametrize("B,H,H_kv,T,n_q", [(64, 32, 32, 16384, 1024), (16, 32, 8, 131072, 512), (32, 32, 8, 16384, 512), (1, 8, 1, 1 << 20, 200),
                                            (1, 8, 1, (1 << 20) + 128, 200), (1, 8, 8, 1 << 24, 200)])
@pytest.mark.parametrize("paged", [False, True])
def test_workspaces_of_4_bit_chunks_are_bounded(B, H, H_kv, T, n_q, paged):
    """What converted rows take: 512 MB and a page table of the requests that are served at a time, whatever the cache's size."""
    d, w = ssa.AttnDesc(), ssa.Window()
    d.B, d.H, d.H_kv, d.D, d.max_ctx, d.kv_dtype, d.out_dtype = B, H, H_kv, 128, T, ssa.FP4_E2M1, ssa.BF16
    d.q_stride_b, d.q_stride_h, d.o_stride_b, d.o_stride_h = H * n_q * 128, n_q * 128, H * n_q * 128, n_q * 128
    for x in "kv":
        setattr(d, x + "_stride_b", 0 if paged else H_kv * T * 128), setattr(d, x + "_stride_h", 128 if paged else T * 128)
        setattr(d, x + "_stride_t", H_kv * 128 if paged else 128)
    w.n_q, w.q_stride_t, w.o_stride_t = n_q, 128, 128
    if paged:
        table = torch.zeros(1, dtype=torch.int32)
        w.paging = C.pointer(ssa.make_paging(table.view(1, 1), 16, 1 << 20))
        w.paging[0].page_table_stride = T // 16
    whole = ssa.attn_window_fp4_workspace_bytes(d, w)
    w.n_q = 32 // (H // H_kv)                                # (few rows: nothing is converted)
    few = ssa.attn_window_fp4_workspace_bytes(d, w)
    assert 0 < few < 1 << 27 and whole > 0
    # partial results: max and sum of every row; and rows of the parts of a context, of as many rows as keep the GPU busy
    rest = B * H * n_q * 8 + (64 << 20)
    converts = T <= 1 << 20                                  # (a head of 2^20 positions is 512 MB)
    assert whole <= rest + converts * ((1 << 29) + B * T // 4)
    assert not converts or whole > 1 << 28
