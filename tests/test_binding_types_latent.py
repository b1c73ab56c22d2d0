"""The calls on a latent cache and the one for rows from logits take the structures and values that they are declared with and nothing that
merely is as long (no GPU needed: the argument is refused before anything is called)."""
import ctypes as C

import pytest
import torch

from paper_2409_10644_amd import binding as b

WRONG = [b.Mlp(), b.AttentionPlan(), (C.c_char * 4096)(), bytearray(4096), None, 7]
T = torch.zeros(8)


@pytest.mark.parametrize("wrong", WRONG, ids=lambda w: type(w).__name__)
def test_another_structure_is_refused(wrong):
    view = b.slice_mask(b.build_mask((2, 2)), 2)
    rope = b.make_rope(0, None)
    for call in (lambda: b.tree_attention_latent(wrong, 1, 4, 512, 64, 0, T, T, 14, T, T, T, 8, 0.1, T, T),
                 lambda: b.tree_latent_norm_rope(wrong, 0, 1, 4, 512, 64, 0, T, T, 8, 8, 8, 8, 8, rope, T, 8, T, T, 14),
                 lambda: b.tree_latent_norm_rope(view, 0, 1, 4, 512, 64, 0, T, T, 8, 8, 8, 8, 8, wrong, T, 8, T, T, 14),
                 lambda: b.store_latent(0, 1, 512, 64, 1, T, 576, 576, wrong, T, T, T, T, 8),
                 lambda: b.sample_rows(0, 1, 1, 8, T, 8, 8, wrong, T, 8, 0, 0, None, None, 0)):
        with pytest.raises((C.ArgumentError, TypeError, AttributeError)):
            call()


def test_settings_of_a_sampler():
    for field, value in (("temperature", torch.zeros(2, dtype=torch.float64)), ("top_k", torch.zeros(2)), ("top_p", torch.zeros(4)[::2]), ("min_p", torch.zeros(2).int())):
        with pytest.raises(b.McsdError):
            b.make_sampler(**{field: value})
    with pytest.raises(b.McsdError):                     # settings of fewer sequences than the call has
        b.sample_rows(0, 3, 1, 8, T, 8, 8, b.make_sampler(torch.ones(2)), T, 8, 0, 0, None, None, 0)
