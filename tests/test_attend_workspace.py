"""Sizes of ecasq_attend's workspace (no GPU): never less for more sequences, keys or heads, so that one made for the largest
sizes serves all smaller ones."""
import itertools


def test_the_size_never_falls():
    from paper_2608_18147_gb300 import native
    size = native.lib().ecasq_workspace_size_attend
    batches = sorted(set(list(range(1, 200)) + [256, 300, 511, 512, 513, 700, 1000, 1216, 1217, 4096, 9728, 9729, 65535]))
    for kv, g, d, n in itertools.product((1, 2, 3, 8, 16), (1, 3, 4, 8, 12), (64, 128, 252), (1, 65, 999, 8192, 100000, 1 << 30)):
        sizes = [size(b, kv * g, kv, d, n) for b in batches]
        assert sizes == sorted(sizes), (kv, g, d, n)
    lengths = sorted({1, 33, 34, 63, 64, 65, 97, 100, 1000, 5000, 99999, 1 << 20, 1 << 30})
    for b, kv, g in itertools.product((1, 7, 100, 128, 700, 3000), (1, 2, 8), (1, 4, 12)):
        sizes = [size(b, kv * g, kv, 128, n) for n in lengths]
        assert sizes == sorted(sizes), (b, kv, g)
    for b, kv, n in itertools.product((1, 50, 100, 128, 700), (1, 2, 8), (65, 5000, 100000)):
        sizes = [size(b, kv * g, kv, 128, n) for g in range(1, 40)]
        assert sizes == sorted(sizes), (b, kv, n)
        more = [size(b, k * 4, k, 128, n) for k in range(1, 40)]
        assert more == sorted(more), (b, n)


def test_the_size_stays_small():
    """It holds as many splits as fill the card a few times, whatever the batch: 8 heads a block, of 8 x 8 x 152 blocks."""
    from paper_2608_18147_gb300 import native
    size = native.lib().ecasq_workspace_size_attend
    for b, kv, g, d in itertools.product((1, 100, 65535), (1, 8, 64), (1, 8, 16), (64, 256)):
        assert size(b, kv * g, kv, d, 1 << 30) <= 8 * 8 * 8 * 152 * (d + 4) * 4
    assert size(65535, 65535, 1, 256, 1 << 30) <= 8 * 8 * 8 * 152 * 260 * 4
