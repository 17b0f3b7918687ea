"""Memory of the 4-bit cache's calls on streams of the caller's choice."""
import numpy as np
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


@pytest.mark.parametrize("rows", [1, 40])
def test_attention_between_its_queries(rows):
    """An output whose rows lie between those of the queries, in one buffer; on the queries it is refused."""
    import torch
    from paper_2510_11331_amd import SDError, attention_q
    from test_gpu_kv_q import Case
    say("output between the queries", rows)
    r = np.random.default_rng(rows)
    H, KV, hd = 4, 2, 64
    c = Case(r, [rows], [100], KV, hd)
    c.fill(r)
    cache = c.cache()
    both = torch.randn(rows, 2 * H, hd, device="cuda").bfloat16()
    q, o = both[:, :H], both[:, H:]
    want = attention_q(q.contiguous(), cache, c.desc)
    kept = q.clone()
    assert attention_q(q, cache, c.desc, out=o).data_ptr() == o.data_ptr() and torch.equal(o, want) and torch.equal(q, kept)
    for out in (q, both[:, 1:H + 1], both[:, H - 1:2 * H - 1]):
        with pytest.raises(SDError):
            attention_q(q, cache, c.desc, out=out)
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(q, kept)
