"""The plain block of a graph network: norm, products and checkpoints in 8 bits run together, against the same block of plain operations."""
import math

import pytest
import torch

import layer_reference as ref
import rows8_reference as ref8
from paper_2106_16064_amd.workloads import rmat_csr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def graph():
    from paper_2106_16064_amd.autograd import SparseOperator
    A = rmat_csr(9, 8, seed=3, values="rownorm")
    dense = torch.zeros(A.M, A.K, dtype=torch.float64)
    rows = torch.repeat_interleave(torch.arange(A.M), torch.as_tensor(A.row_lengths()).long())
    dense[rows, torch.as_tensor(A.colidx).long()] = torch.as_tensor(A.vals).double()
    return SparseOperator(A), dense


def plain(dense, h, t, p, seed, step, activation="gelu"):
    s = h + (ref.dropped(dense @ h, p, seed, step) if p else dense @ h)
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-5) * t["weight"]
    return s, y, s + ref.act(activation, y @ t["w_up"].T + t["b_up"]) @ t["w_down"].T + t["b_down"]


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_block_and_its_gradients(graph, p):
    """In float: eight operations deep, sums of at most 512 terms in each, values below 2^5: 1e-4 is above 8 * 520 * 2^-24 times that over the
    root mean square of a row, which is above 2^-2."""
    from paper_2106_16064_amd.graph_block import PlainBlock
    op, dense = graph
    torch.manual_seed(0)
    block = PlainBlock(24, 40, p, seed=5)
    with torch.no_grad():
        block.b_up.normal_()
        block.b_down.normal_()
    h = torch.randn(dense.shape[1], 24, dtype=torch.float64).float().double()
    on = h.float().cuda().requires_grad_(True)
    out = block(op, on, step=7)
    grad = torch.randn(out.shape, dtype=torch.float64)
    out.backward(grad.float().cuda())
    t = {name: v.detach().double().cpu().requires_grad_(True) for name, v in block.named_parameters()}
    h.requires_grad_(True)
    _, _, want = plain(dense, h, t, p, 5, 7)
    want.backward(grad)
    assert (out.detach().double().cpu() - want.detach()).abs().max() <= 1e-4
    assert (on.grad.double().cpu() - h.grad).abs().max() <= 1e-4 * max(1.0, h.grad.abs().max().item())
    for name, v in block.named_parameters():
        assert (v.grad.double().cpu() - t[name].grad).abs().max() <= 1e-4 * max(1.0, t[name].grad.abs().max().item()), name


def test_activations_in_8_bits_change_the_gradients_as_far_as_they_are_rounded(graph):
    """The result is the same.  Every gradient's error is at most that of its products with x off by amax / 127 / 2 of its block and slopes off by
    1/224: carried through two products that is below a tenth of the gradient in the 2-norm, and the last product's bias has none."""
    from paper_2106_16064_amd.graph_block import PlainBlock
    op, dense = graph
    for dtype in (torch.float32, torch.bfloat16):
        found = {}
        for keep in (False, True):
            torch.manual_seed(1)
            block = PlainBlock(64, 96, 0.1, seed=5, keep_8bit=keep)
            h = torch.randn(dense.shape[1], 64, device="cuda:0").to(dtype).requires_grad_(True)
            grad = torch.randn(dense.shape[0], 64, device="cuda:0").to(dtype)
            out = block(op, h, 3)
            out.backward(grad)
            found[keep] = [out.detach(), h.grad, *(v.grad for v in block.parameters())], [name for name, _ in block.named_parameters()]
        (whole, names), (kept, _) = found[False], found[True]
        assert (whole[0] - kept[0]).abs().max() <= 1e-3 * whole[0].abs().max()                 # the sparse product may add in another order
        for a, b, name in zip(whole[1:], kept[1:], ["h", *names]):
            assert (a.double() - b.double()).norm() <= 0.1 * a.double().norm(), name
        assert torch.equal(whole[1 + 1 + names.index("b_down")], kept[1 + 1 + names.index("b_down")])


def test_serving_form(graph):
    """Against the same steps in 64 bits, with operands rounded to 8 bits where the block rounds them: what is left are borders between two steps that an
    operand's error of 2^-9 (bfloat16) crosses, 2^-3 of an element each, few of a sum."""
    from paper_2106_16064_amd.graph_block import PlainBlock
    op, dense = graph
    torch.manual_seed(2)
    block = PlainBlock(96, 160, 0.0).eval()
    with torch.no_grad():
        block.b_up.normal_()
    t = {name: v.detach().double().cpu() for name, v in block.named_parameters()}
    h = torch.randn(dense.shape[1], 96).bfloat16()
    got = block.in_8bit()(op, h.cuda())
    s, y, whole = plain(dense, h.double(), t, 0.0, 0, 0)
    e4m3 = lambda v: ref8.stands_for(v.float(), "e4m3")  # noqa: E731
    u = ref.act("gelu", e4m3(y) @ e4m3(t["w_up"]).T + t["b_up"]).bfloat16().double()
    want = s + e4m3(u) @ e4m3(t["w_down"]).T + t["b_down"]
    assert got.dtype == torch.bfloat16
    off = (got.double().cpu() - want).norm() / want.norm()
    assert off <= 0.02, off
    assert (got.double().cpu() - whole).norm() <= 0.08 * whole.norm()                            # two products of operands within 2^-4 of themselves
    graph_ = torch.cuda.CUDAGraph()
    serve, on = block.in_8bit(), h.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(op, on)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph_):
        out = serve(op, on)
    for _ in range(3):
        on.mul_(0.5)
        graph_.replay()
        torch.cuda.synchronize()
        assert (out.float() - serve(op, on).float()).norm() <= 0.02 * out.float().norm()
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("keep", [[], ["--keep-8bit"]], ids=["whole", "8bit"])
def test_training_run(dtype, keep):
    from paper_2106_16064_amd.graph_block import main
    losses = main(["--scale", "10", "--width", "32", "--hidden", "64", "--steps", "10", "--dtype", dtype, "--block", "plain", *keep])
    assert len(losses) == 10 and all(math.isfinite(loss) for loss in losses)


def test_checkpoints_in_8_bits_are_of_plain_blocks():
    from paper_2106_16064_amd.graph_block import main
    with pytest.raises(SystemExit):
        main(["--keep-8bit"])
