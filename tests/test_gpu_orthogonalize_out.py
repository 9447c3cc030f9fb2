"""What mf.orthogonalize takes as its output."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_an_output_that_is_no_tensor_is_refused():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf
    g = torch.zeros(2, 6, 8, device="cuda")
    for out in ([1.0], np.zeros((2, 6, 8), np.float32), 3):
        with pytest.raises(mf.MFError) as e:
            mf.orthogonalize(g, out=out)
        assert e.value.status == mf.MF_EINVAL
