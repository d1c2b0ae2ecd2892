"""Lengths of a padded batch that are a slice of a longer list: any first entry, read when the call runs."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [0, 1, 2, 3, 5])
def test_lengths_from_any_place_of_a_list(mw, first):
    """A server keeps one list of lengths and hands out the part of the members at hand."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(first)
    B, H, Hkv, T, M, D = 3, 4, 2, 70, 150, 64
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v, do = rand(B, H, T, D), rand(B, Hkv, M, D), rand(B, Hkv, M, D), rand(B, H, T, D)
    lengths = torch.tensor([150, 33, 0, 64, 149, 1, 90, 7], dtype=torch.int32, device="cuda")
    part = lengths[first:first + B]
    assert part.data_ptr() % 16 == 4 * first % 16

    def run(kv_len):
        o, lse = mw.mw_cross_attn_fwd(q, k, v, kv_len=kv_len)
        return (o, lse, *mw.mw_cross_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len))

    got, want = run(part), run(part.clone())
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(part)
    for turn in range(3):
        lengths.copy_(torch.roll(lengths, 1).clone())
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, run(part.clone())):
            assert torch.equal(a, b)
