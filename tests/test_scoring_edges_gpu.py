"""The label-scoring operators where digits, infinities, autograd's bookkeeping
and sizes at their limits decide: sums that cancel, disallowed labels, states
written in place, large batches."""
import numpy as np
import pytest

import scoringref as R
from test_scoring_gpu import S, gen, labels_of, near, normal  # noqa: F401 (S: the fixture)

pytestmark = pytest.mark.gpu

U64 = 2.0 ** -53


@pytest.mark.parametrize("P,T,V,dtype", [(16, 500, 65, "bfloat16"), (7, 511, 1000, "float32"),
                                         (3, 2001, 40, "float16"), (5, 1, 9, "float32")])
def test_preference_margins_of_near_references(S, P, T, V, dtype):
    """Sequence sums of thousands, references within a few units of them: of the
    log-probabilities (32 bits each) everything is formed in 64 bits and rounded once."""
    import torch
    g = gen(P * T)
    x = normal(g, 2 * P, T, V, dtype=dtype, scale=2.0)
    t = labels_of(g, (2 * P, T), V)
    lp = R.f64(S.label_logprob(x, t))
    L = lp.sum(1)
    ref = (torch.from_numpy(L).cuda() + 5 * normal(g, 2 * P).double()).float()
    loss, seq, margin = S.preference_loss(x, t, ref, beta=0.1)
    off = (T + 8) * U64 * np.abs(lp).sum(1)  # of a sum in 64 bits
    near(seq, L, R.U32 * np.abs(L) * 1.01 + off, "sequences")
    gain, b = L - R.f64(ref), float(np.float32(0.1))
    z = b * (gain[:P] - gain[P:])
    zoff = b * (off[:P] + off[P:]) * 1.01
    near(margin, z, R.U32 * np.abs(z) * 1.01 + zoff, "margin")
    each = np.logaddexp(0, -z)
    near(loss, np.array(each.mean()), R.U32 * each.mean() * 1.01 + zoff.max() + 16 * U64 * each.mean(),
         "loss")
