"""Host side of collecting rows for the small model, no GPU needed."""
from types import SimpleNamespace

import numpy as np
import pytest


def test_rows_before_the_final_norm_are_refused():
    """They are not what the LM head multiplies: a head fitted to them would be fitted to something else. Refused before either model is touched."""
    from paper_2504_07878_amd import adapt, tokroute
    slm = SimpleNamespace(cfg=SimpleNamespace(hidden_tap=tokroute.PRE_FINAL_NORM))
    with pytest.raises(ValueError, match="final norm"):
        adapt.collect(slm, SimpleNamespace(), [[1, 2]], np.zeros((1, 4), np.int32))
