"""The history block's oracle against values worked out by hand, published test vectors and differences."""
import numpy as np

from oracle import history as hs


def test_philox_test_vectors():
    """The three vectors that the generator's authors publish for philox4x32 with 10 rounds."""
    cases = [([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
             ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
             ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
              [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])]
    for counter, key, out in cases:
        assert [int(x) for x in hs.philox([np.uint64(c) for c in counter], key)] == out


def test_dropout_keep():
    keep = hs.dropout_keep(400, 37, 0.25, -5, 2 ** 40 + 3, 7)
    n = keep.size
    assert abs(keep.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / n)
    assert np.array_equal(keep[:50, :20], hs.dropout_keep(50, 20, 0.25, -5, 2 ** 40 + 3, 7))
    for other in [(-4, 2 ** 40 + 3, 7), (-5, 3, 7), (-5, 2 ** 40 + 3, 8), (-5 + 2 ** 32, 2 ** 40 + 3, 7)]:
        assert 0.5 < (keep == hs.dropout_keep(400, 37, 0.25, *other)).mean() < 0.75
    assert hs.dropout_keep(9, 9, 0.0, 1, 1, 0).all() and not hs.dropout_keep(9, 9, 1.0, 1, 1, 0).any()


def test_scan_by_hand():
    gate, value = np.zeros((4, 1)), np.array([[4.0], [8.0], [2.0], [100.0]])
    found = hs.runs(np.array([1, 1, 0, -1]), 4, 2)
    assert found == [(1, 0, 2), (0, 2, 3)]
    out = hs.scan_fwd(gate, value, False, found, np.array([[6.0], [2.0]]), np.zeros((2, 1)))
    assert out["h"][:, 0].tolist() == [3.0, 5.5, 4.0, 0.0] and out["final"][:, 0].tolist() == [4.0, 5.5]
    out = hs.scan_fwd(gate, value, True, hs.runs(None, 4, 2))
    assert out["h"][:, 0].tolist() == [4.0, 10.0, 2.0, 101.0]
    assert hs.sequence_rows([1, 1, 3, 4], 6).tolist() == [-1, 1, 1, 2, -1, -1]


def test_scan_gradients_against_differences():
    rng = np.random.default_rng(0)
    seq = np.array([0, 0, 0, -1, 2, 2, 1])
    found = hs.runs(seq, 7, 3)
    for free in (False, True):
        x = [rng.normal(size=(7, 2)), rng.normal(size=(7, 2)), rng.normal(size=(3, 2))]
        dh, df = rng.normal(size=(7, 2)), rng.normal(size=(3, 2))

        def loss(g, v, h0):
            o = hs.scan_fwd(g, v, free, found, h0, np.zeros((3, 2)))
            return (o["h"] * dh).sum() + (o["final"] * df).sum()

        fwd = hs.scan_fwd(x[0], x[1], free, found, x[2])
        b = hs.scan_bwd(fwd, x[1], free, found, dh, df, np.zeros((3, 2)))
        for n, got in enumerate((b["dgate"], b["dvalue"], b["dinitial"])):
            for i in np.ndindex(got.shape):
                step = np.zeros_like(x[n])
                step[i] = 1e-5
                up, down = ([*x[:n], x[n] + s, *x[n + 1:]] for s in (step, -step))
                assert abs((loss(*up) - loss(*down)) / 2e-5 - got[i]) < 1e-8


def test_expert_sort_by_hand():
    slot, source, offsets, counts = hs.expert_sort([[2, 0], [-1, 2], [2, 5]], 3, 0)
    assert slot.tolist() == [[1, 0], [-1, 2], [3, -1]] and source.tolist() == [1, 0, 3, 4, -1, -1]
    assert offsets.tolist() == [0, 1, 1, 4] and counts.tolist() == [1, 0, 3]
    slot, source, offsets, _ = hs.expert_sort([[2, 0], [-1, 2], [2, 5]], 3, 2)
    assert slot.tolist() == [[4, 0], [-1, 5], [-1, -1]] and source.tolist() == [1, -1, -1, -1, 0, 3]
    assert offsets.tolist() == [0, 2, 4, 6]
