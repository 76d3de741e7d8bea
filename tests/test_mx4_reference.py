"""The numpy reference of the cache in 4 bits, against worked examples."""
import numpy as np

import mx4_reference as M


def test_codes_of_one_block():
    x = np.zeros(32)
    x[:16] = [6, -6, 5, -5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26, 0.24, 5.01, 3.49, 1.74, -0.0]
    code, e = M.encode(x)
    assert e.tolist() == [127]
    want = [6, -6, 4, -4, 4, 2, 2, 1, 1, 0, 0.5, 0, 6, 3, 1.5, 0]
    assert M.decode(code, e)[:16].tolist() == want


def test_exponents():
    for top, e in ((4.0, 127), (6.99, 127), (7.0, 128), (7.99, 128), (8.0, 128), (1.0, 125), (0.0, 2), (1e-40, 2),
                   (2.0 ** 127, 252), (3.4e38, 252), (np.inf, 255), (np.nan, 255)):
        x = np.zeros(32)
        x[7] = top
        assert M.encode(x)[1].tolist() == [e], top
    x = np.zeros(32)
    x[7] = 7.5                                    # 3.75 of the larger scale
    assert M.rounded(x)[7] == 8.0


def test_error_of_a_block():
    """An element is off by at most a fifth of the block's largest magnitude: by the scale, half the
    step from 4 to 6, where it is 5 of it itself; by half of it below 4, which the largest is 3.5 of at least; by less than
    it above 6, where the largest is 7 at most."""
    x = np.random.default_rng(0).normal(size=(2000, 128)) * np.exp2(np.random.default_rng(1).integers(-60, 60, (2000, 1)))
    top = np.abs(x).reshape(2000, 4, 32).max(-1)
    off = np.abs(M.rounded(x) - x).reshape(2000, 4, 32).max(-1)
    assert (off <= top / 5).all()


def test_pages_round_trip():
    rng = np.random.default_rng(3)
    for P in (16, 32):
        for d in (64, 128):
            x = rng.normal(size=(3, P, d))
            for index in (M.key_index(P, d), M.value_index(P, d)):
                assert sorted(index[0].reshape(-1)) == list(range(P * d))
                assert sorted(index[1].reshape(-1)) == list(range(P * d // 2, M.block_bytes(P, d)))
                pages = np.zeros((3, M.block_bytes(P, d)), np.uint8)
                M.put(pages, index, *M.encode(x))
                assert np.array_equal(M.get(pages, index), M.rounded(x))
