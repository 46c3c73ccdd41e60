"""kvb_scan and kvb_scan_backward with so many sequences and v-heads that their workgroups have four or eight waves.  Bounds and inputs are
those of the tests of whole sequences; bf16 sequences and v-heads: 65 to 128 of 128 columns four waves, more eight; of 64 columns four from 129."""
import pytest

from test_gpu_scan import Seqs
from test_gpu_scan_backward import Grads

pytestmark = pytest.mark.gpu

CASES = [
    # lengths, Hk, Hv, d, inputs, outputs
    ([70] * 17, 2, 4, 128, "bf16", "bf16"), ([150, 0, 64, 65] * 6, 2, 4, 128, "bf16", "f32"),       # four waves
    ([70] * 33, 2, 4, 128, "bf16", "f32"), ([200, 70, 0, 64] * 9, 2, 4, 128, "bf16", "bf16"),       # eight
    ([70] * 65, 1, 2, 64, "bf16", "f32"), ([130, 1, 64, 0, 65] * 14, 1, 2, 64, "bf16", "bf16"),     # four, two tiles of columns each way
    ([100] * 43, 1, 3, 128, "bf16", "bf16"),                                                        # 129 with three v-heads a qk-head
]


@pytest.mark.parametrize("lens, Hk, Hv, d, in_dtype, out_dtype", CASES)
def test_outputs_and_states(lens, Hk, Hv, d, in_dtype, out_dtype):
    t = Seqs(lens, Hk, Hv, d, in_dtype, seed=sum(lens) + d)
    t.check(*t.scan(out_dtype), *t.expected(), out_dtype)


@pytest.mark.parametrize("lens, Hk, Hv, d, in_dtype, out_dtype", CASES)
def test_gradients(lens, Hk, Hv, d, in_dtype, out_dtype):
    Grads(lens, Hk, Hv, d, in_dtype, seed=sum(lens) + d, out_dtype=out_dtype).check_backward()


def test_rows_of_one_projection_and_a_gap_in_front():
    for lens, Hk, Hv, d in (([70, 130, 0] * 12, 2, 4, 128), ([90, 64] * 33, 1, 2, 64)):
        t = Grads(lens, Hk, Hv, d, "bf16", seed=3, gap=37, fused=True)
        t.check(*t.scan(), *t.expected())
        t.check_backward()
