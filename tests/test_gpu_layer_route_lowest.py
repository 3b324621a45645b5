"""sdp_route on the GPU with biases at the ends of FP32: a bias of the lowest value masks
an expert without taking it out, and sums of two such are numbers still."""
import pytest

from test_gpu_layer_route import BF16, F32, check, ctx, logits  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LOW = torch.finfo(torch.float32).min


def biases(e, groups, gen):
    """Masked experts by the lowest value, in some groups all of them, and large biases of either sign."""
    each = e // groups
    some = 0.1 * torch.randn(e, generator=gen)
    yield torch.full((e,), LOW)
    last = some.clone()
    last[each:] = LOW
    yield last
    for low in (LOW, 0.7 * LOW, -LOW, -0.7 * LOW):
        masked = some.clone().view(groups, each)
        masked[::2] = low
        masked[1, :] = low
        masked[1, 0] = 0.0
        yield masked.view(-1)
    mixed = some.clone()
    mixed[::3], mixed[1::3] = LOW, -LOW
    yield mixed
    gone = last.clone()
    gone[:each // 2] = float("-inf")
    yield gone


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("e,groups,top_groups,top", [(8, 4, 4, 7), (16, 4, 3, 9), (64, 8, 8, 8), (64, 8, 4, 8), (24, 2, 1, 2),
                                                     (256, 8, 4, 8), (96, 6, 6, 20), (60, 5, 3, 6)])
def test_biases_of_the_lowest_value(ctx, e, groups, top_groups, top, sigmoid):  # noqa: F811
    gen = torch.Generator().manual_seed(e + top)
    for dtype in (F32, BF16):
        z = logits(20, e, dtype, e)
        z[3, ::2] = float("-inf")
        for bias in biases(e, groups, gen):
            for best in (1, 2):
                check(ctx, z, top, bias.cuda(), sigmoid, groups, top_groups, best)
            check(ctx, z, top, bias.cuda(), sigmoid)
