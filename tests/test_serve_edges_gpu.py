"""The long-context operators on the GPU where they are used less often: on
other streams, near the ends of the numbers' range, with odd records and
arguments.  Against the plain 64-bit statement (tests/serve_ref.py)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import serve_ref  # noqa: E402
import synth  # noqa: E402
from gpu_util import say  # noqa: E402
from test_window_gpu import Case  # noqa: E402

pytestmark = pytest.mark.gpu

mlkv = pytest.importorskip("paper_2406_09297_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    mlkv.lib()
    yield


@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("four_bits", [True, False])
def test_split_runs_on_another_stream(four_bits, as_handle):
    """Units of two runs beside units of one, merged on a stream that was never
    used before: every row is written, from counters that were zero, and they are
    zero again.  Of a bare handle the caller orders the fill of `out`."""
    say(f"split runs on another stream four_bits={four_bits} handle={as_handle}")
    lens = [33] * 40 + [3000]
    c = Case(four_bits, 12, 4, 64, lens, 3040, 53, k_scale=3.0)
    want = c.decode(hint=3000)
    assert not c.ws[:262144].any()
    side = torch.cuda.Stream()
    f = mlkv.qcache_decode_attention if four_bits else mlkv.decode_attention_window
    for _ in range(3):
        out = torch.full(c.q.shape, 7.0, device="cuda")
        if as_handle:
            side.wait_stream(torch.cuda.current_stream())
        f(c.layer, c.q, c.cache, c.map, c.seq_lens, out, window=0, max_len_hint=3000, ws=c.ws,
          stream=side.cuda_stream if as_handle else side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)
        assert not c.ws[:262144].any()
