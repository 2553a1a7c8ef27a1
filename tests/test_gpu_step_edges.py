"""GPU tests of a decoding step's operators where a formula's ends meet: lists
that overflow, sums that are rounded on their way, the last bits of a product,
weights that are not finite.  Tolerances are derived where they stand."""
import numpy as np
import pytest

from tests.test_gpu_step import check_tokens, dev, gen, host, rows_of, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,fp32", [(6000, True), (16377, False), (24001, True), (32760, True)])
def test_sample_short_rows_with_long_lists(V, fp32):
    """Rows of few groups in which more elements stay than the list holds: they are counted
    once, found too many, and counted again."""
    import paper_2608_00916_amd as moe
    B = 70
    say("sample long lists", V, fp32)
    logits = rows_of(B, V, V + 1, fp32)
    g = gen(V)
    u = dev(g.random(B).astype(np.float32))
    p = dev(g.choice([0.9, 0.99, 0.999], B).astype(np.float32))
    t = dev(g.choice([1.0, 2.0, 8.0], B).astype(np.float32))
    m = dev(g.choice([1e-9, 1e-6, 1e-3], B).astype(np.float32))
    op, few = moe.Sampler(B, V), moe.Sampler(3, V)
    for s in (dict(temperature=t, top_p=p), dict(temperature=t, min_p=m), dict(temperature=t, top_p=p, min_p=m)):
        say("  ", list(s))
        token, logprob = (o.clone() for o in op.forward(logits, u, **s))
        check_tokens(logits, u, (token, logprob), **s)
        for _ in range(5):
            again = op.forward(logits, u, **s)
            assert (again[0] == token).all() and (again[1] == logprob).all()
        some = few.forward(logits[9:12], u[9:12], **{n: v[9:12] for n, v in s.items()})
        assert (some[0] == token[9:12]).all() and (some[1] == logprob[9:12]).all()
