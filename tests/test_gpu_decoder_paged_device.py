"""The decoder over paged caches refuses caches on another device than its weights'."""
import pytest
import torch

from paper_2608_15383_amd._lib import EMOE_EINVAL, ExactMoEError
from tests.test_gpu_decoder import SMALL, _model
from tests.test_gpu_decoder_paged import Paged

pytestmark = pytest.mark.gpu


def test_caches_elsewhere():
    p = Paged(SMALL, _model(SMALL, seed=1))
    first = p.run([5], [0], [0])
    p.dec.device = torch.device("cuda:1")      # as if the weights were there
    with pytest.raises(ExactMoEError) as e:
        p.run([5], [0], [0])
    assert e.value.status == EMOE_EINVAL and "cuda:1" in str(e.value)
    p.dec.device = torch.device("cuda:0")
    assert (p.run([5], [0], [0])[0] == first[0]).all()
    p.close()
