"""Memory that two entries of an AdamW step share: one launch would write both, so a
tied weight given twice, or views and states that overlap, are refused before any."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_entries_that_share_memory_are_refused(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    tied, flat = f(300), f(4000)
    for params in ([tied, tied], [tied, f(8), tied], [flat[:2000], flat[1999:]],
                   [flat[100:200], flat], [f(8), flat, f(8), flat[3999:]],
                   # an entry inside one, and one that starts before the first's end
                   [flat[:3000], flat[3000:3100], flat[2990:2995]]):
        with pytest.raises(ValueError, match="shares memory"):
            sgc.AdamW(params)
    m, v = f(300), f(300)
    for states in ({"exp_avgs": [m, m], "exp_avg_sqs": [v, f(300)]},
                   {"exp_avgs": [m, v], "exp_avg_sqs": [v, f(300)]},
                   {"exp_avgs": [m, f(300)], "exp_avg_sqs": [v, m]}):
        with pytest.raises(ValueError, match="shares memory"):
            sgc.AdamW([f(300), f(300)], states=states)
    p = [f(300), f(300)]
    with pytest.raises(ValueError, match="shares memory"):
        sgc.AdamW(p, states={"exp_avgs": [m, p[0]], "exp_avg_sqs": [v, f(300)]})
    scales = f(8)
    codes = {"exp_avgs": [f(300, dtype=torch.int8) for _ in p],
             "exp_avg_sqs": [f(300, dtype=torch.uint8) for _ in p]}
    with pytest.raises(ValueError, match="shares memory"):
        sgc.AdamW(p, state_bits=8, states=codes | {
            "exp_avg_scales": [scales[:2], scales[2:4]],
            "exp_avg_sq_scales": [scales[4:6], scales[3:5]]})


def test_neighbours_are_taken(gpu):
    """Entries side by side in one buffer, in any order, empty ones among them."""
    import paper_2507_23387_amd as sgc

    for order in itertools.permutations(range(4)):
        flat = torch.ones(1000, device="cuda")
        cuts = (0, 300, 300, 301, 1000)
        params = [flat[cuts[i]:cuts[i + 1]] for i in order]
        opt = sgc.AdamW(params, lr=0.5, weight_decay=0.0)
        opt.step([torch.ones_like(p) for p in params])
        assert torch.all((flat - 0.5).abs() <= 1e-6)
