"""The gated quantizer to 8 bits where its workgroups hold the table, in every shape of them: rows aligned and not, and, where a call may have more rows than workgroups run at once, so many that some
take a second and a third one."""
import numpy as np
import pytest
import torch

from oracle import grouped
from paper_2506_04985_amd import binding as fptq
from test_gpu_quantize8 import guarded_codes, host, rows, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K", [(3200, 505), (7300, 504), (7301, 505), (1600, 1000), (7300, 1000), (7301, 1001), (2900, 1800), (2901, 1801), (800, 3000), (801, 3001), (1900, 3000), (1901, 3001),
                                 (2000, 5000), (2000, 5001), (3000, 5001), (250, 7000), (251, 7001), (900, 7000), (901, 7001), (1100, 8000), (1100, 8001), (2100, 8001), (1100, 11000),
                                 (1100, 11001), (1100, 14336), (1101, 14001), (250, 14336), (251, 14001), (600, 20000), (600, 20001), (600, 28000), (600, 28001)])
def test_gated(M, K):
    g = torch.Generator(device="cuda").manual_seed(M * 11 + K)
    gate, up = rows(g, M, 2 * K).split(K, 1)
    whole, out = guarded_codes(M, K)
    codes, scale = fptq.fptq_gated_quantize8(gate, up, out=out)
    want, want_scale = grouped.quantize_rows(grouped.gated(host(gate), host(up)))
    assert untouched(whole)
    assert np.array_equal(codes.cpu().numpy(), grouped.lay_out(want))
    assert np.array_equal(scale.cpu().numpy(), want_scale)
