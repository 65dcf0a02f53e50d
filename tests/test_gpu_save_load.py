"""What is brought back into a decoder's pages has to go with it: nothing is planned for rows that do not."""
import pytest

pytestmark = pytest.mark.gpu

PROMPTS = [[5, 6], [17, 4, 4, 250, 17], [(7 * i * i + 3) % 300 for i in range(70)]]


def _decoder(**over):
    import torch
    from paper_2603_14110_amd.draft import random_decoder

    made = dict(layers=2, V=300, dtype=torch.bfloat16, requests=len(PROMPTS), pages=24, page=32, max_len=256, bias=1e4)
    return random_decoder(**{**made, **over})


@pytest.mark.parametrize("bad", ["type", "layers", "heads", "tokens", "requests", "lengths", "host", "lists"])
def test_rows_that_do_not_go_with_a_decoder_change_nothing(bad):
    import torch

    a = _decoder()
    a.prefill(PROMPTS)
    lens, k, v = a.save()
    b = _decoder()
    wrong = {"type": (lens, k.float(), v.float()), "layers": (lens, k[:1], v[:1]), "heads": (lens, k[:, :, :1], v[:, :, :1]), "tokens": (lens, k[:, 1:], v[:, 1:]),
             "requests": (lens[:2], k[:, :sum(lens[:2])], v[:, :sum(lens[:2])]), "lengths": ([lens[0] + 5, -5, sum(lens) - lens[0]], k, v),
             "host": (lens, k.cpu(), v.cpu()), "lists": (lens, k, v[:, :-1])}[bad]
    with pytest.raises(ValueError, match="go with"):
        b.load(wrong)
    assert b.lens.tolist() == [0] * len(PROMPTS) and int(b.pool[1]) == b.ring.numel()
    b.load((lens, k, v))
    assert b.lens.tolist() == lens
    for want, got in zip((k, v), b.save()[1:]):
        assert torch.equal(want, got)
