"""The calls that Python refuses, with device memory: the native half declines each of them first, and the words are the same."""
import pytest
import torch

from test_cache_binding import _calls
from test_cache_refusals import ALL, REFUSED

pytestmark = pytest.mark.gpu


def _on_gpu(x):
    if isinstance(x, torch.Tensor):
        return x.cuda()
    return tuple(_on_gpu(t) for t in x) if isinstance(x, (tuple, list)) else x


@pytest.mark.parametrize("name,i", ALL)
def test_refused(lantern_gpu, name, i):
    change, kind, words = REFUSED[name][i]
    kw = {key: _on_gpu(x) for key, x in _calls()[name].items()}
    kw.update(change(kw))
    with pytest.raises(kind) as e:
        getattr(lantern_gpu, name)(**kw)
    assert words in str(e.value), str(e.value)


@pytest.mark.parametrize("name", REFUSED)
def test_the_right_call_goes_through(lantern_gpu, name):
    kw = {key: _on_gpu(x) for key, x in _calls()[name].items()}
    getattr(lantern_gpu, name)(**kw)
    torch.cuda.synchronize()
