"""Page numbers of a sequence's table that are no pages: every such number is reported, whichever it is."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_attend import KINDS, call, check, make, reference  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,levels", KINDS)
@pytest.mark.parametrize("page", [16, 32, 9])
def test_every_bad_page_number_is_reported(page, dtype, levels):
    import paper_2608_18147_gb300 as E
    c = make([100, 77], 2, 2, 64, page, dtype, levels, seed=page)
    good = c["table"].clone()
    leave = {(0, t) for t in range(page, 2 * page)}
    want = reference(dict(c, table=good), leave=leave)
    pages = c["k"].rows.shape[0]
    for number in (-1, -2, -3, -2 ** 31, pages, 2 ** 31 - 1):
        c["table"][0, 1] = number
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = call(c, status=status)
        assert status.item() == E.BAD_PAGE, number
        check(got, want)
    c["table"][0, 1] = good[0, 1]
    c["table"][1, -(-77 // page):] = -2  # beyond a sequence's end nothing is looked at
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(c, status=status)
    assert status.item() == 0
