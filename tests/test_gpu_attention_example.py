"""The example that takes a compressed prompt through an attention layer: the
macro-tokens of the pass, prefill at their positions and decoding behind them."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("workload", ["tiny"])
def test_prefill_and_decode_behind_a_compressed_prompt(workload):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import attention_layer
    import workloads as WL
    import paper_2607_19368_gb300 as sls
    w = WL.WORKLOADS[workload]
    M, far = attention_layer.run(workload, steps=5)
    assert M == sls.output_count(sls.Config.make(rho=w.rho, D=w.D, r=w.r, bits=w.bits,
                                                 preserve_last=w.preserve_last), w.N)
    # bfloat16 activations: each side rounds queries, keys, weights and outputs once
    # (2^-8 each), and the projections' products may round differently with the row count
    assert max(far) <= 6 * 2.0 ** -8, far
