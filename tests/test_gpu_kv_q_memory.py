"""Memory of the 4-bit cache's calls on streams of the caller's choice."""
import pytest

from sdcase import say

pytestmark = pytest.mark.gpu


def test_rope_table_on_a_stream():
    """Its memory is neither in use by the current stream nor given away there before it is written."""
    import torch
    from paper_2510_11331_amd import rope_table
    say("rope table on a stream")
    n_pos, hd = 3000, 128
    side = torch.cuda.Stream()
    want = rope_table(n_pos, hd)
    for _ in range(3):
        # dropped before its stream has come to it
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        rope_table(n_pos, hd, stream=side)
        other = [torch.full_like(want, 7.0) for _ in range(4)]
        torch.cuda.synchronize()
        assert all(x.eq(7.0).all() for x in other)
        # taken while the current stream still reads what was there
        torch.cuda._sleep(20_000_000)
        copies = [x.clone() for x in other]
        del other
        tables = [rope_table(n_pos, hd, stream=side) for _ in range(4)]
        torch.cuda.synchronize()
        assert all(x.eq(7.0).all() for x in copies) and all(torch.equal(x, want) for x in tables)
        del copies, tables
