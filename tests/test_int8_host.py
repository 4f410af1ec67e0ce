"""Host side of the 8-bit integer calls: what the binding refuses before a call reads out of a matrix.  No GPU needed."""
import pytest
import torch

from paper_2603_19172_amd import binding as B


def call(name, *a, **kw):
    class Fake:
        _h, device = None, 0
    return getattr(B.Context, name)(Fake(), *a, stream=0, **kw)


def pair(n, k, device="cpu"):
    return (torch.zeros((-(-n // 32) * 32, -(-k // 128) * 128), dtype=torch.int8, device=device), torch.zeros(n, device=device))


def expert(H, F, device="cpu"):
    return [pair(F, H, device), pair(F, H, device), pair(H, F, device)]


def test_experts_of_other_sizes_than_the_tables_are_refused():
    table = B.make_int8_table([expert(200, 40), None, expert(200, 40)], "cpu")
    ffn = lambda H, F, t: call("moe_ffn_int8", torch.zeros(4, H), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), t, F)
    for H, F in ((200, 41), (200, 8000), (201, 40), (40, 200)):
        with pytest.raises(ValueError, match="the table's experts"):
            ffn(H, F, table)
    with pytest.raises(ValueError, match="context is of device"):       # the table's own sizes: only the tensors' device is wrong here
        ffn(200, 40, table)
    # a table that the caller made says nothing of sizes, but holds whole entries
    with pytest.raises(ValueError, match="context is of device"):
        ffn(200, 41, torch.zeros((3, 6), dtype=torch.int64))
    for bad in (torch.zeros(100, dtype=torch.uint8), torch.zeros(0, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="whole entries"):
            ffn(200, 40, bad)


def test_tables_refuse_pointers_that_a_kernel_could_not_follow():
    other = expert(200, 40, "meta")
    for bad in ([other], [expert(200, 40), other], [expert(200, 40)[:2] + other[2:]], [[(c, s.to("meta")) for c, s in expert(200, 40)]]):
        with pytest.raises(ValueError, match="device"):
            B.make_int8_table(bad, "cpu")
    for i in range(3):
        ex = expert(200, 40)
        codes, scale = ex[i]
        flat = torch.zeros(codes.numel() + 16, dtype=torch.int8)
        for off in (1, 8):
            ex[i] = (flat[off:off + codes.numel()].view(codes.shape), scale)
            with pytest.raises(ValueError, match="16-byte"):
                B.make_int8_table([ex], "cpu")
        ex[i] = (flat[16:].view(codes.shape), scale)
        assert B.make_int8_table([ex], "cpu").numel() == 48
