"""Host-side refusals of the token sampler, and its oracle's own properties (no GPU needed)."""
import math

import numpy as np
import pytest
import torch

from oracle import np_sample
from paper_2412_01034_b200 import _lib, api, build

A = 0x10000   # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def test_sample_validation(lib):
    def f(x=A, type=0, ld=100, u=A, t=A, k=A, p=A, m=A, out=A, B=2, V=100):
        return lib.qil_sample(x, type, ld, u, t, k, p, m, out, B, V, None)

    for kw in (dict(x=None), dict(u=None), dict(t=None), dict(out=None)):
        assert f(**kw) == 1, kw
    for kw in (dict(B=0), dict(V=0), dict(ld=-1), dict(B=-1), dict(V=-5), dict(B=(1 << 27) + 1)):
        assert f(**kw) == 2, kw
    for kw in (dict(x=0x10002), dict(x=0x10001, type=1), dict(u=0x10002), dict(t=0x10001), dict(k=0x10002), dict(p=0x10002), dict(m=0x10002), dict(out=0x10002)):
        assert f(**kw) == 3, kw
    for kw in (dict(type=3), dict(V=262145, ld=262145)):
        assert f(**kw) == 4, kw


def test_the_binding_refuses_wrong_tensors(lib):
    good = dict(logits=torch.zeros(2, 8), u=torch.zeros(2), temperature=torch.ones(2), top_k=torch.zeros(2, dtype=torch.int32), top_p=torch.ones(2),
                min_p=torch.zeros(2), out=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        api.sample(**good)
    for name, bad in (("logits", torch.zeros(2, 8, dtype=torch.float64)), ("logits", torch.zeros(8)), ("u", torch.zeros(3)), ("temperature", 1.0),
                      ("top_k", torch.zeros(2)), ("top_p", torch.ones(2, dtype=torch.float64)), ("min_p", torch.ones(1)), ("out", torch.zeros(2))):
        with pytest.raises(ValueError):
            api.sample(**dict(good, **{name: bad}))
    for name in ("u", "temperature", "top_k", "top_p", "min_p", "out"):
        with pytest.raises(ValueError, match=f"{name} is on meta"):
            api.sample(**dict(good, **{name: good[name].to("meta")}))


def test_oracle_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert np_sample.pick(x, 0.05, 1.0)[0] == 0 and np_sample.pick(x, 0.3, 1.0)[0] == 1 and np_sample.pick(x, 0.99, 1.0)[0] == 3
    assert np_sample.distribution(x, 1.0, top_k=2)[0].tolist() == [1, 3]
    assert np_sample.distribution(x, 1.0, top_p=0.6)[0].tolist() == [1, 3]
    assert np_sample.distribution(x, 1.0, top_p=0.75)[0].tolist() == [1, 2, 3]
    assert np_sample.distribution(x, 1.0, min_p=0.6)[0].tolist() == [1, 3]
    assert np_sample.distribution(x, 0.0)[0].tolist() == [1]
    assert np_sample.distribution(np.zeros(5), 1.0, top_k=2)[0].tolist() == [0, 1]
    assert np_sample.pick(np.full(3, -math.inf), 0.5, 1.0)[0] == -1
