"""CPU: tensors that the kernels of packed attention would read as something else, or beyond their end, are refused before
anything reaches a GPU."""
import pytest
import torch

import paper_2410_19367_amd as bp

LAYOUT = dict(tokens=100, sequences=3, heads=8, kv_heads=2, head_dim=64, causal=True)
ADDRESSES = [4096] * 5


class OnDevice(torch.Tensor):
    """A host tensor that says it lies in device memory: for what is refused after that check, and what is taken."""
    is_cuda = True


def on_device(t):
    return t.as_subclass(OnDevice)


def refused(call, *words):
    with pytest.raises(bp.BitPipeError) as e:
        call()
    assert e.value.code == bp.BP_EINVAL
    for w in words:
        assert w in str(e.value)


@pytest.mark.parametrize("starts", [torch.tensor([0, 10, 30, 100]), torch.tensor([0.0, 10, 30, 100]), torch.tensor([0, 10, 30, 100], dtype=torch.int16),
                                    torch.tensor([0, 10, 30], dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2],
                                    torch.tensor([0, 10, 30, 100], dtype=torch.int32).numpy(), [0, 10, 30, 100]])
def test_starts_refused(starts):
    """int64 is what cumsum gives: as int32 it is other sequences."""
    refused(lambda: bp.bp_packed(starts=on_device(starts) if isinstance(starts, torch.Tensor) else starts, **LAYOUT), "starts")


def test_host_memory_refused():
    refused(lambda: bp.bp_packed(starts=torch.zeros(4, dtype=torch.int32), **LAYOUT), "device memory")
    refused(lambda: bp.bp_relpos(32, 128, torch.zeros(32, 8)), "device memory")


@pytest.mark.parametrize("table", [torch.zeros(32, 8, dtype=torch.float64), torch.zeros(32, 8, dtype=torch.bfloat16), torch.zeros(31),
                                   torch.zeros(8, 32).t(), torch.zeros(32, 8).numpy()])
def test_table_refused(table):
    refused(lambda: bp.bp_relpos(32, 128, on_device(table) if isinstance(table, torch.Tensor) else table), "table")


def test_table_and_its_gradient_of_too_few_heads_refused():
    layout = bp.bp_packed(starts=4096, **LAYOUT)
    small = bp.bp_relpos(32, 128, on_device(torch.zeros(32, 4)))
    fine = bp.bp_relpos(32, 128, 4096)

    def bwd(bias, dtable=None):
        return bp.bp_op_attention_packed_bwd(bp.BP_BF16, layout, *ADDRESSES, *[4096] * 4, 4096, bias=bias, dtable=dtable, workspace_elems=1)

    refused(lambda: bp.bp_op_attention_packed_fwd(bp.BP_BF16, layout, *ADDRESSES, bias=small), "[32, 8]")
    refused(lambda: bwd(small), "[32, 8]")
    for dtable in (torch.zeros(32, 4), torch.zeros(32, 8, dtype=torch.bfloat16), torch.zeros(8, 32).t()):
        refused(lambda: bwd(fine, on_device(dtable)), "dtable")
    refused(lambda: bwd(fine), "workspace")


def test_workspace_counts_bytes():
    """A workspace of two-byte elements has room for half as many floats as it has elements."""
    layout = bp.bp_packed(starts=4096, **LAYOUT)
    n = bp.bp_op_attention_packed_workspace(bp.BP_BF16, layout)
    assert n > 0
    least = 100 * 8
    ws = torch.zeros(2 * least - 8, dtype=torch.bfloat16)
    refused(lambda: bp.bp_op_attention_packed_bwd(bp.BP_BF16, layout, *ADDRESSES, *[4096] * 4, ws), "workspace")


def test_what_is_right_is_taken():
    starts = on_device(torch.tensor([0, 10, 30, 100, 100], dtype=torch.int32))
    table = on_device(torch.zeros(32, 8))
    layout, bias = bp.bp_packed(starts=starts, **LAYOUT), bp.bp_relpos(32, 128, table)
    assert layout.starts == starts.data_ptr() and bias.table == table.data_ptr()
    assert bp.bp_op_attention_packed_workspace(bp.BP_BF16, layout, bias) > 0


@pytest.mark.parametrize("sequences", [1 << 24, (1 << 31) - 64, (1 << 31) - 1])
def test_more_sequences_than_tokens_can_be_refused(sequences):
    layout = bp.bp_packed(starts=4096, **{**LAYOUT, "sequences": sequences})
    assert bp.bp_op_attention_packed_workspace(bp.BP_BF16, layout) == 0
    for call in (lambda: bp.bp_op_attention_packed_fwd(bp.BP_BF16, layout, *ADDRESSES),
                 lambda: bp.bp_op_attention_packed_bwd(bp.BP_BF16, layout, *ADDRESSES, *[4096] * 4, 4096, workspace_elems=1 << 30)):
        with pytest.raises(bp.BitPipeError) as e:
            call()
        assert e.value.code == bp.BP_ESHAPE
    assert bp.bp_op_attention_packed_workspace(bp.BP_BF16, bp.bp_packed(starts=4096, **{**LAYOUT, "sequences": (1 << 24) - 1})) > 0


def test_pointers_to_the_structures_are_taken():
    """As ctypes takes them: refused for what they point at only."""
    import ctypes as C
    layout, bias = bp.bp_packed(starts=4096, **LAYOUT), bp.bp_relpos(32, 3, 4096)
    for b in (C.byref(bias), C.pointer(bias), bias):
        refused(lambda: bp.bp_op_attention_packed_fwd(bp.BP_BF16, C.byref(layout), *ADDRESSES, bias=b), "max_distance")
        refused(lambda: bp.bp_op_attention_packed_bwd(bp.BP_BF16, C.byref(layout), *ADDRESSES, *[4096] * 4, 4096, bias=b, dtable=4096,
                                                      workspace_elems=1 << 30), "max_distance")
