"""The status word of the operators on 4-bit codes: an int32 tensor on the device, of any shape; its first element is the word."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def calls():
    import paper_2608_18147_gb300 as E
    idx = torch.randint(0, 16, (8, 128), dtype=torch.uint8, device="cuda")
    product = (torch.randn(128, device="cuda"), E.ecasq_pack(idx), torch.randn(16, device="cuda"), torch.rand(8, 4, device="cuda"), 32)
    rows = torch.randn(2, 16, 1, 32, device="cuda")
    table, lengths = torch.tensor([[7, 0]], dtype=torch.int32, device="cuda"), torch.tensor([20], dtype=torch.int32, device="cuda")
    codes = torch.zeros(2, 16, 1, 16, dtype=torch.uint8, device="cuda")
    levels = torch.zeros(2, 16, 1, 8, device="cuda").half()
    write = (torch.randn(1, 1, 32, device="cuda"), torch.zeros(1, 8, device="cuda"), None, torch.tensor([99], device="cuda"), codes, levels, 1)
    return [(lambda s: E.ecasq_matvec(*product, status=s), 0), (lambda s: E.ecasq_cache_write(*write, status=s), E.BAD_PAGE),
            (lambda s: E.ecasq_attend(torch.randn(1, 2, 32, device="cuda"), rows, rows, table, lengths, status=s), E.BAD_PAGE)]


@pytest.mark.parametrize("shape", [(), (1,), (3,), (1, 1), (2, 1, 1, 1, 2)])
def test_any_shape(shape):
    for call, bits in calls():
        status = torch.zeros(shape, dtype=torch.int32, device="cuda")
        call(status)
        assert status.view(-1)[0].item() == bits and not status.view(-1)[1:].any()


def test_an_element_of_a_larger_tensor():
    for call, bits in calls():
        words = torch.zeros(4, dtype=torch.int32, device="cuda")
        call(words[2])
        assert words.tolist() == [0, 0, bits, 0]


def test_refusals():
    import paper_2608_18147_gb300 as E
    for call, _ in calls():
        for wrong in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int64, device="cuda"), 0,
                      torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")):
            with pytest.raises(E.EcasqError, match="status"):
                call(wrong)
