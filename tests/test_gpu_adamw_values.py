"""What AdamW.state_values returns: float32 tensors in the parameters' shapes, with
32-bit states views of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(3, 5), (7,), (2, 3, 4), (0, 4), ()]


@pytest.mark.parametrize("bits", [32, 8])
def test_shapes(gpu, bits):
    import paper_2507_23387_amd as sgc

    opt = sgc.AdamW([torch.ones(s, device="cuda") for s in SHAPES], state_bits=bits)
    for _ in range(2):
        opt.step([torch.ones(s, device="cuda") for s in SHAPES])
        for values in opt.state_values():
            assert [tuple(t.shape) for t in values] == SHAPES
            assert all(t.dtype == torch.float32 for t in values)
            assert all((t > 0).all() for t in values)


def test_32_bit_values_are_the_states(gpu):
    import paper_2507_23387_amd as sgc

    states = {"exp_avgs": [torch.zeros(15, device="cuda")],
              "exp_avg_sqs": [torch.zeros((5, 3), device="cuda")]}
    opt = sgc.AdamW([torch.ones((3, 5), device="cuda")], states=states)
    (m,), (v,) = opt.state_values()
    opt.step([torch.ones((3, 5), device="cuda")])
    for value, key in ((m, "exp_avgs"), (v, "exp_avg_sqs")):
        assert value.shape == (3, 5) and value.data_ptr() == states[key][0].data_ptr()
        assert torch.equal(value.view(-1), states[key][0].view(-1)) and (value > 0).all()
