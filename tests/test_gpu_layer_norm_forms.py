"""Every form that the layer norm and its backward pass are launched in, by rows on an SM and columns of a row, against the oracle in 64 bits:
blocks that go from row to row, and shares whose rows go round the places that they are copied ahead to more than twice.  The bounds are
those of the tests of the operators."""
import pytest

from paper_2510_25590_b200 import binding
from test_gpu_layer_norm import Case, _backward, _check_backward, _check_forward, _forward, _ragged

pytestmark = pytest.mark.gpu


def _sms():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


def _case(rows, C, groups, residual, modulated=True):
    return Case(rows, C, _ragged(rows, groups), groups, residual=residual, modulated=modulated)


# rows (of an SM), columns: eight warps to a row, four, two, one; one to four pieces of a row to a thread
FORWARD = [(3, 1000), (3, 2056), (10, 4104), (10, 8192),
           (13, 1000), (13, 1536), (13, 2560), (13, 4096), (17, 2056), (17, 4096),
           (20, 1032), (20, 1536), (20, 1544), (20, 2048), (70, 1032), (70, 2048),
           (70, 200), (70, 264), (70, 704), (70, 1000)]


@pytest.mark.parametrize("each,C", FORWARD)
@pytest.mark.parametrize("residual", [False, True])
def test_forward_forms(each, C, residual):
    c = _case(each * _sms() + 5, C, 7, residual)
    _check_forward(c, _forward(c))


# rows of an SM, columns, whether the gated residual is there: one piece of a row to a thread (four rows of a team on their way, and nine of a team
# in a share), then two (three, and seven); rows of one to eight teams
BACKWARD = [(72, 264, True), (36, 1000, True), (18, 2048, True), (9, 4096, True), (9, 2304, True), (16, 2048, False), (9, 4096, False), (15, 1032, False),
            (7, 4104, True), (7, 8192, True), (7, 4104, False), (7, 8192, False), (56, 264, False), (56, 1000, False), (28, 2048, False), (17, 4096, False)]


@pytest.mark.parametrize("each,C,residual", BACKWARD)
@pytest.mark.parametrize("groups,dz", [(5, True), (41, False)])
def test_backward_forms(each, C, residual, groups, dz):
    c = _case(each * _sms() + 11, C, groups, residual)
    _check_backward(c, _backward(c, dz), dz)


def test_backward_of_a_buffer_with_more_rows_than_live_ones():
    """The launch is chosen for the rows of the buffer, the shares for those of the ranges."""
    rows = 40 * _sms()
    c = Case(rows, 1000, [(3, rows // 3), (rows // 2, rows // 2 + 1), (rows // 2 + 4, rows // 2 + 600)], 3, residual=True, modulated=True)
    _check_backward(c, _backward(c, True), True)


def test_backward_workspace_of_a_wider_call_does():
    """The size that is asked for is enough whichever form is taken: a byte less is refused, and nothing behind it is written."""
    import torch
    rows = 20 * _sms()
    c = _case(rows, 1000, 6, False)
    n = binding.layer_norm_backward_workspace(rows, 6, 1000)
    held = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    _check_backward(c, _backward(c, True, workspace=held[:n]), True)
    assert torch.all(held[n:] == 77)
    with pytest.raises(binding.RegionEError):
        _backward(c, True, workspace=held[:n - 1])
