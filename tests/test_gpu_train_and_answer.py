"""The 4-bit training example: rounding, update and products run together as a program uses them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state_bits", [8, 32])
def test_it_learns_and_answers(state_bits):
    from paper_2504_20634_b200 import train_and_answer
    first, last, answered, zero = train_and_answer.run(steps=300, state_bits=state_bits)
    assert last < 0.5 * first                                   # it learns
    assert answered < 1.2 * last + 0.02 * zero                  # and answers, with bfloat16 tokens, about as well as it trained


def test_answers_are_the_product_of_the_rounded_values():
    from paper_2504_20634_b200 import train_and_answer
    net = train_and_answer.FourBitNetwork(200, 136, seed=3)
    net.round(1)
    token = torch.randn(200, device="cuda").to(torch.bfloat16)
    h = torch.relu(net.values[0].double() @ token.double()).to(torch.bfloat16)
    want = net.values[1].double() @ h.double()
    got = net.answer(token).double()
    # the hidden layer may differ by one bfloat16 unit where the sums' rounding decides
    assert float((got - want).norm()) < 2.0 ** -7 * float(want.norm())
