"""The two forms of the loss's gradient (a draft row in one workgroup; behind the loss's launch, which q' rows ask for) where float32 has no
room for what the row's temperatures and masks make of its logits: both against the oracle and against ot_distill_loss."""
import numpy as np
import pytest

from test_gpu_distill_grad import MODES, _compare, _spec
from workloads import make_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_qprime", [False, True])
@pytest.mark.parametrize("V_d", [301, 9001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiny_draft_temperatures(dtype, V_d, with_qprime):
    """Above and below the temperature from which a row is done in 64 bits; masked draft ids, whose exponent is the largest."""
    temps = [1.0, 3e-8, 2e-8, 5e-9, 4e-9, 1e-12, 1e-30, 1e-36]
    case = make_case(_spec("tiny_draft", [5, 3, 6, 4, 4, 7, 2, 5], 41, dtype=dtype, V_t=max(600, V_d), V_d=V_d, temperature=[1.0] * 8, draft_temperature=temps))
    low = np.float32(-np.inf) if dtype == "f32" else np.uint16(0xFF80)
    out = np.random.default_rng(2).random(case.draft_logits.shape) < 0.3
    out[np.arange(case.K), case.draft_ids] = False
    case.draft_logits[out] = low
    _compare(case, modes=MODES, with_qprime=with_qprime)


@pytest.mark.parametrize("with_qprime", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiny_target_temperatures(dtype, with_qprime):
    """ln p down to -1e31, which the gradient follows."""
    temps = [1.0, 3e-8, 2e-8, 1e-9, 1e-20, 1e-30]
    case = make_case(_spec("tiny_target", [5, 3, 6, 4, 4, 7], 43, dtype=dtype, temperature=temps, draft_temperature=[1.0, 0.7, 1.0, 1.0, 0.5, 1.0]))
    _compare(case, modes=MODES, with_qprime=with_qprime)
