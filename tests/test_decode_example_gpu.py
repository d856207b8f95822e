"""The example that runs the decoding operators together."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("requests,drafts,dtype", [(4, 16, torch.float16), (1, 1, torch.bfloat16), (9, 40, torch.bfloat16)])
def test_tree_steps_equal_single_steps(requests, drafts, dtype):
    """A row passes five products and an attention whose inputs and results
    are rounded to the type, each in another order of sums: six roundings of a
    unit roundoff, doubled by the two additions, on values of up to five times
    the root mean square."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("speculative_step", os.path.join(ROOT, "examples", "speculative_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    worst = example.run(requests=requests, steps=2, drafts=drafts, dtype=dtype, width=512, heads=8, key_heads=2, hidden=1024)
    assert worst <= 6 * 2 * 5 * (2.0 ** -11 if dtype is torch.float16 else 2.0 ** -8)
