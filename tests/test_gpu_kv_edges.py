"""The 8-bit key/value cache where sizes, values or events are out of the
ordinary; the bounds are those of test_gpu_kv.py."""
import pytest
from test_gpu_kv import check_attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,new,typ", [(128, 20, "bf16"), (96, 32, "f16"), (256, 12, "bf16"), (192, 30, "f16")])
def test_attend_large_batches_of_many_rows(cuda_ok, d, new, typ):
    """1024 sequences take more shared memory beside a large tile than a CTA has: several launches."""
    check_attend(1, 1, d, 16, typ, [(i % 23, new - i % 3) for i in range(1024)])
