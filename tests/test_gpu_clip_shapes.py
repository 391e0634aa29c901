"""A list's tensors and their outputs of different shapes: what a pair may look like is the pair's own matter."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_clip import check, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("strided", ["tensor", "out", "both"])
def test_reshaped_outputs_beside_rows_apart(strided):
    """Contiguous outputs of as many values, next to a matrix of rows apart from each other and on its own."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"clip reshaped {strided}")
    gen = torch.Generator("cuda").manual_seed(7)
    make = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    tensors = [make(4, 8), make(5, 6, 7), make(33)]
    outs = [torch.zeros(8, 4, device="cuda"), torch.zeros(210, device="cuda"), torch.zeros(3, 11, device="cuda")]
    ws, norm = workspace(readout, torch, 4), torch.empty(1, device="cuda")
    readout.clip(tensors, 0.5, norm, ws, out=outs)
    check(torch, tensors, [o.reshape(t.shape) for t, o in zip(tensors, outs)], norm, 0.5)
    wide = [torch.full((9, 20), float("nan"), device="cuda") for _ in range(2)]
    apart, to = (w[:, 2:15] for w in wide)
    apart.copy_(make(9, 13))
    if strided == "out":
        apart = apart.contiguous()
    if strided == "tensor":
        to = torch.zeros(9, 13, device="cuda")
    for o in outs:
        o.zero_()
    readout.clip([*tensors, apart], 0.5, norm, ws, out=[*outs, to])
    check(torch, [*tensors, apart], [*(o.reshape(t.shape) for t, o in zip(tensors, outs)), to], norm, 0.5)
    if strided != "tensor":
        assert int(wide[1].isnan().sum()) == 9 * 7


def test_pairs_that_do_not_match_are_refused():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("clip pairs refused")
    ws, norm = workspace(readout, torch, 2), torch.empty(1, device="cuda")
    flat, wide = torch.ones(4, 8, device="cuda"), torch.ones(9, 20, device="cuda")[:, 2:15]
    for tensors, out in (([flat], [torch.ones(4, 9, device="cuda")]), ([flat, wide], [torch.ones(4, 9, device="cuda"), torch.ones(9, 13, device="cuda")]),
                         ([flat, wide], [flat.clone(), torch.ones(13, 9, device="cuda")]), ([flat, wide], [flat.clone(), torch.ones(117, device="cuda")]),
                         ([flat, wide.contiguous()], [flat.clone(), torch.ones(13, 20, device="cuda")[:, :9]]), ([flat, wide], [flat.bfloat16(), torch.ones(9, 13, device="cuda")]),
                         ([flat, wide], [flat.clone(), wide.contiguous().bfloat16()])):
        with pytest.raises(ValueError, match="out"):
            readout.clip(tensors, 1.0, norm, ws, out=out)
    assert bool((flat == 1).all()) and bool((wide == 1).all())
