"""Keys and values that are infinite or NaN and seen: what the definition makes
of them, element by element.  A score of -Inf has weight 0; one of +Inf or NaN
makes its row of that head NaN; a value of Inf or NaN reaches its own element of
the outputs alone."""

import numpy as np
import pytest
import torch

from . import latent_ref
from .gpu_util import say
from .latent_ref import check
from .prompt_ref import DROP, HIGH, LOW, f64

pytestmark = pytest.mark.gpu
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
from .test_gpu_prompt import Run, normal  # noqa: E402

INF, NAN = float("inf"), float("nan")
N = 300


class Both:
    """A cache of HIGH entries holding k and v as they are, and the reference with zeros in the odd places."""

    def __init__(self, D, k, v, window=0, actions=(HIGH,)):
        self.r = Run(1, 4, 2, D, 400, actions, seed=1, window=window)
        self.r.s.append(0, None, k.cuda(), v.cuda(), keep_all=True)
        self.k, self.v = f64(torch.nan_to_num(k[0], 0, 0, 0)), f64(torch.nan_to_num(v[0], 0, 0, 0))

    def run(self, q):
        out = torch.full((1, *q.shape), -77.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((1, *q.shape[:2]), -77.0, device="cuda")
        say("attend", tuple(q.shape))
        self.r.s.prompt(0, q[None].cuda(), out, lse)
        torch.cuda.synchronize()
        return f64(out[0]), f64(lse[0])

    def want(self, q, h, gone=()):
        """Out, lse and bounds of head h; `gone`: tokens of weight 0."""
        n, g = len(q), h * 2 // 4
        seen = np.arange(N)[None] <= N - n + np.arange(n)[:, None]
        seen[:, list(gone)] = False
        return latent_ref.attention(f64(q[:, h]), self.k[:, g], self.v[:, g], self.r.s.softmax_scale, seen)


def tensors(seed, D, n_q):
    g = torch.Generator().manual_seed(seed)
    return normal(g, 1, N, 2, D), normal(g, 1, N, 2, D), normal(g, n_q, 4, D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [4, 120])
@pytest.mark.parametrize("gone", [(0, 100), (0, 1), (40, 41), (32, 170), (290, 300), (0, 300)])
def test_scores_of_minus_infinity_have_no_weight(D, n_q, gone):
    """One key, and runs of them that fill whole steps of the kernels, whose scores for two of the heads are -Inf."""
    k, v, q = tensors(D + n_q, D, n_q)
    gone = range(*gone)
    k[0, gone.start:gone.stop, 0, 3] = -INF
    q[:, :2, 3] = q[:, :2, 3].abs() + 0.5
    b = Both(D, k, v)
    out, lse = b.run(q)
    for h in range(4):
        if h < 2 and len(gone) == N:
            assert (np.isnan(out[:, h]) | (out[:, h] == 0)).all()      # no weight at all: 0 / 0, or nothing seen
            continue
        want, want_lse, tol, lse_tol = b.want(q, h, gone if h < 2 else ())
        check(out[:, h], want, tol, f"out of head {h}")
        check(lse[:, h], want_lse, lse_tol, f"lse of head {h}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [4, 120])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("key", [INF, NAN])
@pytest.mark.parametrize("at", [0, 100, N - 3])
def test_infinite_and_nan_scores_reach_their_rows_alone(D, n_q, window, key, at):
    """NaN from the token on in the heads that read it, whole rows and lse; the other heads and the rows before it exact."""
    k, v, q = tensors(D + n_q + 1, D, n_q)
    k[0, at, 0, 3] = key
    q[:, :2, 3] = q[:, :2, 3].abs() + 0.5
    b = Both(D, k, v, window)
    out, lse = b.run(q)
    m = max(0, at - (N - n_q))                        # queries before the token
    for h in range(4):
        want, want_lse, tol, lse_tol = b.want(q, h)
        end = m if h < 2 else n_q
        check(out[:end, h], want[:end], tol[:end], f"out of head {h}")
        check(lse[:end, h], want_lse[:end], lse_tol[:end], f"lse of head {h}")
        assert np.isnan(out[end:, h]).all() and np.isnan(lse[end:, h]).all(), f"head {h}"


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [4, 120])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_values_reach_their_own_element(D, n_q, window, value):
    k, v, q = tensors(D + n_q + 2, D, n_q)
    at = N - 2
    v[0, at, 1, 7] = value
    b = Both(D, k, v, window)
    out, lse = b.run(q)
    m = at - (N - n_q)
    for h in range(4):
        want, want_lse, tol, lse_tol = b.want(q, h)
        check(lse[:, h], want_lse, lse_tol, f"lse of head {h}")
        if h >= 2:
            got = out[m:, h, 7]
            assert np.isnan(got).all() if np.isnan(value) else (got == value).all(), got
            out[m:, h, 7] = want[m:, 7]
        check(out[:, h], want, tol, f"out of head {h}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [4, 120])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("at", [0, 100])
def test_values_that_all_queries_see_reach_their_own_element(D, n_q, value, at):
    """Among whole steps of keys: that element of the heads that read it is not finite, every other one exact."""
    k, v, q = tensors(D + n_q + 3, D, n_q)
    v[0, at, 1, 7] = value
    out, lse = (b := Both(D, k, v)).run(q)
    for h in range(4):
        want, want_lse, tol, lse_tol = b.want(q, h)
        check(lse[:, h], want_lse, lse_tol, f"lse of head {h}")
        if h >= 2:
            assert not np.isfinite(out[:, h, 7]).any()
            out[:, h, 7] = want[:, 7]
        check(out[:, h], want, tol, f"out of head {h}")
