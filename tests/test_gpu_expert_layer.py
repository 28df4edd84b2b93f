"""The expert operators around the device-resident AllToAllv: tokens of R ranks to their experts and back."""
import pytest
import torch

from paper_2608_00358_b200 import experts as ex
from paper_2608_00358_b200.expert_layer import ExpertParallel

pytestmark = pytest.mark.gpu


def make(R, k, tokens, hidden, inner, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    up, down = torch.randn(R, inner, hidden, device="cuda", generator=g), torch.randn(R, hidden, inner, device="cuda", generator=g)
    layer = ExpertParallel(ex.Router(R, k), [ex.Int8Linear.from_float(up[e:e + 1]) for e in range(R)],
                           [ex.Int8Linear.from_float(down[e:e + 1]) for e in range(R)], tokens, act=torch.relu)
    x = [torch.randn(tokens, hidden, device="cuda", generator=g).bfloat16() for _ in range(R)]
    skew = torch.linspace(1.5, -1.5, R, device="cuda")
    logits = [torch.randn(tokens, R, device="cuda", generator=g) + skew for _ in range(R)]
    return layer, ex.Int8Linear.from_float(up), ex.Int8Linear.from_float(down), x, logits


def alone(router, up, down, x, logits):
    """The same on one rank that holds all experts: no exchange."""
    r = router.route(logits)
    h = torch.relu(up(x, routing=r))
    return ex.combine(down(h, offsets=r.offsets), r)


@pytest.mark.parametrize("R,k,tokens,hidden,inner", [(2, 1, 5, 64, 96), (8, 2, 100, 256, 512), (8, 8, 33, 128, 128), (16, 3, 1, 200, 136), (70, 4, 20, 64, 64)])
def test_exchanged_experts_give_the_bits_of_experts_in_one_place(R, k, tokens, hidden, inner):
    layer, up, down, x, logits = make(R, k, tokens, hidden, inner)
    for turn in range(2):  # the second pass has other counts in the same buffers
        y = layer.forward(x, logits)
        layer.check()
        for r in range(R):
            assert torch.equal(y[r], alone(layer.router, up, down, x[r], logits[r])), (turn, r)
        logits = [t.flip(0).roll(1, 1).contiguous() for t in logits]


def test_a_pass_replays_from_a_graph():
    layer, up, down, x, logits = make(4, 2, 24, 128, 256)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer.forward(x, logits)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        y = layer.forward(x, logits)
    for _ in range(3):
        for t in logits:
            t.copy_(t.roll(1, 1))
        graph.replay()
        layer.check()
        for r in range(4):
            assert torch.equal(y[r], alone(layer.router, up, down, x[r], logits[r]))
