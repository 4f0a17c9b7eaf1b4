"""CPU-only checks of what the binding of caches, attention and logits refuses before a kernel is given a pointer."""
import pytest
import torch

import paper_1804_10112_amd as spt

i32 = lambda *a: torch.tensor(a, dtype=torch.int32)


def _words(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


@pytest.mark.parametrize("mask", [_words(1, 100).expand(8, 100), _words(8, 1).expand(8, 100), _words(300).as_strided((8, 100), (20, 1)),
                                  _words(8, 200)[:, ::2], _words(100, 8).t(), _words(8), _words(8, 100).long()],
                         ids=["one row for all", "one word for all", "overlapping rows", "every other word", "words apart", "one axis", "int64"])
def test_masks_whose_rows_lie_otherwise_are_refused(mask):
    """The kernel reads row r at r * stride, so a stride below the words of a row would be read as another one."""
    with pytest.raises(spt.SptError):
        spt.LogitRules(first=i32(0, 8), allowed=mask)


@pytest.mark.parametrize("mask,stride", [(_words(8, 100), 100), (_words(8, 200)[:, 50:150], 200), (_words(1, 100), 100),
                                         (_words(4, 200)[:1, 10:90], 80), (_words(8, 1), 1), (_words(8, 7)[:, 3:4], 7)])
def test_strides_of_masks(mask, stride):
    assert spt.LogitRules(first=i32(0, 8), allowed=mask).c.allowed_stride == stride


def test_a_mask_with_too_few_words_for_the_vocabulary_is_refused():
    """Whatever its stride: the bits behind a row's last word are another tensor's."""
    logits = torch.zeros(8, 321)
    rules = spt.LogitRules(first=i32(0, 8), allowed=_words(8, 200)[:, :10])
    with pytest.raises(spt.SptError, match="words"):
        spt.spt_adjust_logits(logits, rules, torch.empty_like(logits))
