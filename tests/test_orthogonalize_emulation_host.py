"""That what the orthogonalised updates are held to sees mistakes: each is planted in
the emulation, on the CPU, and has to be refused, and the emulation itself not."""
import pytest
import torch

import orthogonalize_emulation as E

BF, F32 = torch.bfloat16, torch.float32
# with operands in pairs a X and the diagonal may as well be in the product, single operands have no mixed one
NONE_OF_PAIRS, NONE_OF_SINGLES = ("diagonal in the product", "a X in the product"), ("mixed product dropped",)


@pytest.mark.parametrize("rows,cols", [(150, 300), (320, 200)])
@pytest.mark.parametrize("spread", [True, False])
def test_mistakes_in_pairs_are_seen(rows, cols, spread):
    u = E.make(rows, cols, F32, spread=spread)
    held = E.Held(u, F32, True)
    assert held.why_not(E.emulate(u, True, exact_sums=True)) is None and held.why_not(held.exact) is None
    missed = [m for m in E.MISTAKES if held.why_not(E.emulate(u, True, mistake=m)) is None]
    assert missed == [m for m in E.MISTAKES if m in NONE_OF_PAIRS]


def test_mistakes_in_single_operands_are_seen():
    u = E.make(150, 300, BF)
    held = E.Held(u, BF, False)
    assert held.why_not(E.emulate(u, False, exact_sums=True)) is None and held.why_not(held.exact) is None
    missed = [m for m in E.MISTAKES if held.why_not(E.emulate(u, False, mistake=m)) is None]
    assert missed == list(NONE_OF_SINGLES)


@pytest.mark.parametrize("rows,cols", [(63, 65), (96, 200), (500, 520)])
def test_gross_mistakes_in_single_operands_are_seen_at_any_size(rows, cols):
    u = E.make(rows, cols, BF)
    held = E.Held(u, BF, False)
    for m in ("zeros", "four steps", "b off by 1%", "bf16 operands"):
        assert held.why_not(E.emulate(u, False, mistake=m))


def test_a_wrong_block_of_a_large_answer_is_seen():
    """One of 64 blocks of 64 x 64 with the neighbour's values, or 30 times its error."""
    for dtype, pairs in ((F32, True), (BF, False)):
        u = E.make(500, 520, dtype)
        held = E.Held(u, dtype, pairs)
        x = held.near.clone()
        x[448:, 192:256] += 30 * (held.offs[0] / x.numel() ** 0.5) * torch.randn(52, 64, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
        assert held.why_not(x)
        x = held.near.clone()
        x[192:256, :64] = x[192:256, 64:128].clone()
        assert held.why_not(x)
