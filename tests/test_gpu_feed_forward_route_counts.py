"""iroute_top's counts of a chunk of tokens, in 8 and in 16 bits: as many as fit, few experts folded over the lanes, more chunks than the 256 that are wanted."""
import pytest
import torch

from paper_2006_11735_amd import binding as B

pytestmark = pytest.mark.gpu


def check(logits, top):
    """Against torch's stable sorts; gates are left to the other tests"""
    rows, experts = logits.shape
    d = B.route_desc(rows=rows, experts=experts, top=top, normalise=1)
    many = rows * top
    new = lambda *shape: torch.full(shape, -7, dtype=torch.int32, device="cuda:0")  # noqa: E731
    expert, place, token, offsets, gate = new(rows, top), new(rows, top), new(many), new(experts + 1), torch.zeros((rows, top), device="cuda:0")
    ws = torch.full((B.iroute_top_workspace_bytes(d),), 0xEE, dtype=torch.uint8, device="cuda:0")
    B.iroute_top(d, logits, expert, gate, place, token, offsets, ws)
    torch.cuda.synchronize()
    want = torch.empty_like(expert)
    for at in range(0, rows, 1 << 20):
        want[at:at + (1 << 20)] = torch.sort(logits[at:at + (1 << 20)], dim=1, descending=True, stable=True).indices[:, :top].int()
    assert torch.equal(expert, want)
    flat = want.reshape(-1)
    order = torch.sort(flat, stable=True).indices
    assert torch.equal(token, (order // top).int())
    to = torch.empty(many, dtype=torch.int32, device="cuda:0")
    to[order] = torch.arange(many, dtype=torch.int32, device="cuda:0")
    assert torch.equal(place.reshape(-1), to)
    bounds = torch.searchsorted(flat[order].contiguous(), torch.arange(experts + 1, dtype=torch.int32, device="cuda:0"))
    assert torch.equal(offsets, bounds.int())


@pytest.mark.parametrize("rows", [57344, 57345, 65536, 65537, 70001])   # the most tokens that are counted in 8 bits: 256 chunks of 224
@pytest.mark.parametrize("experts,top", [(3, 2), (8, 2), (12, 3), (16, 16), (20, 2), (24, 5), (30, 2), (32, 4), (40, 2), (48, 6), (64, 1), (65, 2), (256, 8), (1000, 3)])
def test_counts_of_8_and_of_16_bits(rows, experts, top):
    g = torch.Generator(device="cuda:0").manual_seed(rows + experts)
    check(torch.randn((rows, experts), generator=g, device="cuda:0"), top)
    check(torch.zeros((rows, experts), device="cuda:0"), top)              # (every token's are the first experts)
    last = torch.zeros((rows, experts), device="cuda:0")
    last[:, -1] = 1
    check(last, top)


@pytest.mark.parametrize("rows", [1 << 23, (1 << 23) + 1, (1 << 23) + 40000, 20000003])      # chunks of 32768 tokens, the largest: 256 of them and more
@pytest.mark.parametrize("experts,top", [(6, 2), (33, 1)])
def test_chunks_of_the_largest_size(rows, experts, top):
    g = torch.Generator(device="cuda:0").manual_seed(rows)
    check(torch.randn((rows, experts), generator=g, device="cuda:0"), top)
    check(torch.zeros((rows, experts), device="cuda:0"), top)
