"""The tests' own generator against the vectors its authors publish with it (kat_vectors, philox4x32 10)."""
import numpy as np

import dropout_ref as dr


def word(text):
    return [int(w, 16) for w in text.split()]


def test_known_answers():
    for counter, key, want in (("0 0 0 0", "0 0", "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
                               ("ffffffff ffffffff ffffffff ffffffff", "ffffffff ffffffff", "408f276d 41c83b0e a20bc7c6 6d5451fd"),
                               ("243f6a88 85a308d3 13198a2e 03707344", "a4093822 299f31d0", "d16cfe09 94fdcceb 5001e420 24126ea1")):
        got = dr.philox([np.array([v], dtype=np.uint64) for v in word(counter)], word(key))
        assert [int(v) for v in got[:, 0]] == word(want)


def test_thresholds():
    assert [dr.cut_of(p) for p in (0.0, 0.1, 0.5, 1.0, 1e-6)] == [0, 6554, 32768, 65536, 0]
