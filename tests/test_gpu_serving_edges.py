"""The serving operators at their edges: settings that are no number, values that are not finite, queries with one large channel, prompts that fill
the append's tiles, recorded and eager steps in turn, calls that are refused before anything is written."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from test_gpu_serving import (DEV, DTYPE, KINDS, attend_case, check_append, check_attention, check_sample, check_tables, dev, host, make_pool, paged_step,
                              pool_to_dev)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- the paged step

def test_decode_step_refuses_other_numbers_of_tokens():
    from paper_2504_12285_b200 import chain as gpu_chain
    from paper_2504_12285_b200 import workloads as wl
    from test_gpu_serving import small_layers

    table = torch.zeros(500, 256, dtype=torch.bfloat16, device=DEV)
    st = gpu_chain.DecodeStep(small_layers(1, 256, 512, 128, 8700), table, 2, 64, 256, 512, 4, 2, 64, wl.RMS_EPS, device=DEV)
    for n in (1, 3):
        with pytest.raises(ValueError):
            st.step(torch.zeros(n, dtype=torch.int32, device=DEV))
    assert st.step(torch.zeros(2, dtype=torch.int32, device=DEV)).shape == (2, 500)
