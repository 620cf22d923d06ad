"""The words that say that a bounded wait of an attention kernel ran out.  They are set here by the host, as a kernel would."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_the_word_of_prompts_is_cleared_by_the_check():
    q = torch.randn((8, 2, 64), device=DEV).bfloat16()
    cu = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    disc.disc_attend_prompt(q, q, q, cu, max_len=8)
    disc.disc_attend_check()
    disc.model_ops._error_word(q.device).fill_(1)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_check()
    disc.disc_attend_check()
