"""One workspace, made for the largest batch and length, serves every smaller call."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_attend import call, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("levels", [0, 8])
def test_a_batch_that_shrinks_keeps_its_workspace(levels):
    import paper_2608_18147_gb300 as E
    hkv, g, d, n = 8, 2, 64, 6000
    most = 130
    c = make([n - 17 * i for i in range(most)], hkv, g, d, 16, "bf16", levels, seed=5)
    ws = E.workspace_attend(most, hkv * g, hkv, d, c["table"].shape[1] * 16)
    for b in (130, 128, 113, 100, 77, 50, 31, 12, 3, 1):
        part = dict(c, q=c["q"][:b], table=c["table"][:b], lengths=c["lengths"][:b])
        for max_len in (None, n, 999):
            got, want = (call(part, max_len=max_len, ws=w) for w in (ws, None))
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
