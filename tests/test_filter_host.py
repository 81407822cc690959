"""Refusals of the filtered operators that need no GPU, and the definitions' plain form against worked numbers."""
import numpy as np

from filter_plain import Row, draw, verify
from paper_2506_03700_amd import binding as ad


def test_null_arguments():
    L = ad.lib()
    f = ad.Filter(1.0, 0, 0.0, 0.0)
    assert L.ad_filtered_probs(None, None, 1, f, None, None) == ad.AD_EINVAL
    assert L.ad_sample_filtered(None, None, f, 0.5, None, None, None) == ad.AD_EINVAL
    assert L.ad_sample_filtered_wait(None, None, f, 0.5, None, None, None) == ad.AD_EINVAL
    assert L.ad_verify_filtered(None, None, None, None, 1, f, None, None, 0.5, None, None, None, None) == ad.AD_EINVAL
    assert L.ad_verify_filtered_wait(None, None, None, None, 1, f, None, None, 0.5, None, None, None, None) == ad.AD_EINVAL
    assert L.ad_generate_filtered(None, None, None, 0, None, None, None, None, None, None, 0, None, None) == ad.AD_EINVAL


def test_worked_rows():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.2, 0.1]))
    p = lambda *f: Row(z.astype(np.float32), 1.0, *f).p
    np.testing.assert_allclose(p(0, 0.0, 0.0), [0.1, 0.4, 0.2, 0.2, 0.1], rtol=1e-6)
    np.testing.assert_allclose(p(2, 0.0, 0.0), [0, 2 / 3, 1 / 3, 0, 0], rtol=1e-6)          # equal ones: the lower id
    np.testing.assert_allclose(p(0, 0.5, 0.0), [0, 2 / 3, 1 / 3, 0, 0], rtol=1e-6)
    np.testing.assert_allclose(p(0, 0.61, 0.0), [0, 0.5, 0.25, 0.25, 0], rtol=1e-6)
    np.testing.assert_allclose(p(3, 0.7, 0.0), [0, 2 / 3, 1 / 3, 0, 0], rtol=1e-6)          # 0.7 of the three's 0.8 is 0.56
    np.testing.assert_allclose(p(0, 0.0, 0.45), [0, 0.5, 0.25, 0.25, 0], rtol=1e-6)
    assert draw(p(0, 0.61, 0.0), 0.6)[0] == 2 and draw(p(0, 0.61, 0.0), 0.0)[0] == 1
    P, Q = [Row(z.astype(np.float32), 1.0, 2)] * 2, [Row(z.astype(np.float32), 1.0, 1)]
    assert verify(P, Q, [1], [0.6], [0.5], 0.9)[:2] == (1, 2)                               # ratio 2/3
    assert verify(P, Q, [1], [0.7], [0.5], 0.9)[:2] == (0, 2)                               # what is left is id 2
