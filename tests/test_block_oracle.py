"""The plain definitions of the norms, the dropout and the sequences' losses against what is known of them: published outputs of the generator, closed forms, and
gradients by differences."""
import numpy as np
import pytest

from oracle import block_oracle as ob


def test_generator_known_answers():
    """Counters and keys with the outputs that the generator's authors publish for 4 words, 32 bits, 10 rounds."""
    f = 0xFFFFFFFF
    cases = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
             ((f, f, f, f), (f, f), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
             ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for c, k, want in cases:
        assert tuple(int(x) for x in ob.philox(c, k)) == want
        assert tuple(int(x) for x in ob._philox_fast(*c, *k)) == want


def test_mask():
    """The places of the half-words, and the share of what is kept: 65536 - 6554 of 65536 for p = 0.1; 200000 values: a deviation of 0.00067."""
    seed, step, site = (7 << 32) + 5, (3 << 32) + 9, 4
    m = ob.keep(3, 19, 0.1, seed, step, site)
    for r in range(3):
        for c in range(19):
            w = int(ob.philox(((c // 8) + (site << 16), r, 9, 3), (5, 7))[c % 8 // 2])
            assert m[r, c] == ((w >> 16 if c & 1 else w & 0xFFFF) >= 6554)
    big = ob.keep(100, 2000, 0.1, 11, 12, 0)
    assert abs(big.mean() - (65536 - 6554) / 65536) < 5 * 0.00067
    assert (ob.keep(100, 2000, 0.1, 11, 13, 0) != big).any() and (ob.keep(100, 2000, 0.1, 11, 12, 1) != big).any()
    assert ob.keep(4, 50, 0.0, 1, 2, 3).all() and ob.threshold(0.1) == 6554


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_gradients_by_differences(kind):
    r = np.random.RandomState(1)
    z, w, b, dy = r.randn(3, 7), r.randn(7), r.randn(7), r.randn(3, 7)
    f = lambda z, w, b: (ob.norm_fwd(z, w, b, kind, 1e-3)[0] * dy).sum()  # noqa: E731
    y, mean, rstd, h = ob.norm_fwd(z, w, b, kind, 1e-3)
    dz, dw, db = ob.norm_bwd(dy, h, rstd, w, kind)
    for x, got, at in ((z, dz, 0), (w, dw, 1), (b, db, 2)):
        for i in np.ndindex(x.shape):
            args = [[z.copy(), w.copy(), b.copy()] for _ in range(2)]
            for a, sign in zip(args, (1, -1)):
                a[at][i] += sign * 1e-5
            diff = (f(*args[0]) - f(*args[1])) / 2e-5
            assert abs(diff - got[i]) < 1e-7 * (1 + abs(diff))   # the third derivative's term is of the order 1e-10, the cancellation's 1e-11


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_seq_loss_gradients_by_differences(gate):
    r = np.random.RandomState(2)
    T, E, k = 9, 5, 2
    x = r.randn(T, E)
    topk = np.argsort(-x, 1)[:, :k]
    ranges = [(0, 3), (3, 3), (4, 8)]
    counts, P, loss, dz = ob.seq_loss(x, topk, ranges, k, gate, 0.3, 0.2)
    assert counts.sum() == k * 7 and counts[1].sum() == 0 and np.allclose(P.sum(1), [1, 0, 1]) and not dz[[3, 8]].any()
    for i in np.ndindex(x.shape):
        both = []
        for sign in (1, -1):
            y = x.copy()
            y[i] += sign * 1e-5
            both.append(ob.seq_loss(y, topk, ranges, k, gate, 0.3, 0.2)[2].sum())
        assert abs((both[0] - both[1]) / 2e-5 - dz[i]) < 1e-9 + 1e-7 * abs(dz[i])


def test_seq_loss_of_balanced_loads():
    """Uniform scores: P = 1 / E, so the balance is alpha whatever the loads; lse = log E."""
    E, T = 4, 8
    topk = np.array([[t % E] for t in range(T)])
    _, P, loss, dz = ob.seq_loss(np.zeros((T, E)), topk, [(0, 4), (4, 8)], 1, "softmax", 0.5, 0.25)
    assert np.allclose(P, 1 / E) and np.allclose(loss, [0.5, 0.25 * np.log(E) ** 2]) and np.allclose(dz, 2 * 0.25 / T * np.log(E) / E)
