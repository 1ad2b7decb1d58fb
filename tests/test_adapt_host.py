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


def test_no_entries():
    """Rows for cross entropy alone: nothing of the teacher is listed."""
    import torch
    from paper_2504_07878_amd import adapt, tokroute
    out = lambda *a, **k: SimpleNamespace(hidden=torch.ones(2, 8), logits=torch.zeros(2, 10))   # noqa: E731
    slm = SimpleNamespace(cfg=SimpleNamespace(hidden_tap=tokroute.POST_FINAL_NORM), prefill=out, decode_step=out)
    llm = SimpleNamespace(shape=dict(vocab=10), device="cuda:0", prefill=out, decode_step=out)
    hidden, ids, teacher, targets = adapt.collect(slm, llm, [[1, 2], [3]], np.arange(6, dtype=np.int32).reshape(2, 3), top=0)
    assert hidden.shape == (6, 8) and ids.shape == teacher.shape == (6, 0) and ids.dtype == torch.int32 and targets.tolist() == [0, 3, 1, 4, 2, 5]
