"""The gated delta rule's plan without a GPU: what its workspace holds."""
import ctypes

from test_abi_host import mb  # noqa: F401  (the loaded library)
from test_sequence_host import attention


def test_no_room_for_cuts_that_cannot_be(mb):  # noqa: F811
    """A sequence is cut where it is longer than two shares of the rows: of one or two shares none is, so a call with so many
    heads that no more come out needs no room for states and maps of parts."""
    bytes_of = mb.load().mmbev_gated_delta_workspace_bytes
    size = lambda heads, back=0, n=1: bytes_of(ctypes.byref(attention(  # noqa: E731
        mb, rows=100000, num_sequences=n, max_length=0, heads=heads, kv_heads=heads, key_dim=128, value_dim=128, dtype=0)), back)
    assert size(128) == 256 and size(86) == 256 and size(85) == 256 and size(64, n=3) == 256  # one share, and two
    assert size(64) > 3 * 64 * 128 * 128 * 8  # three
    # backwards the chunks' states and rows alone
    chunks, rows = (100000 // 32 + 1) * 128 * 128 * 128 * 4, 100000 * 128 * 128 * 4
    assert 0 <= size(128, 1) - 2 * (chunks + rows) < 4 * 256


def test_parts_for_the_workgroups_that_fit(mb):  # noqa: F811
    """A long sequence of 8 heads is cut so that its parts fill the chip's 256 units once: four workgroups a unit in bf16, three
    in fp16, whose rows take more LDS, but of heads up to 32 four; the room is proportional to the parts."""
    def room(dtype, dim):
        return mb.load().mmbev_gated_delta_workspace_bytes(ctypes.byref(attention(mb, rows=120000, num_sequences=1, heads=8, kv_heads=8, key_dim=dim,
                                                                                  value_dim=64, dtype=dtype)), 0)

    for dtype, dim, parts in ((2, 64, 127), (1, 64, 95), (1, 40, 95), (0, 64, 63)):
        one = 8 * dim * (64 + 2 * dim) * 4  # a state and two maps
        assert parts * one < room(dtype, dim) < (parts + 1) * one + 16 * 8 * dim * 64 * 4, (dtype, dim)
    assert room(1, 32) == room(2, 32)
