"""What bm_add_adapters' binding refuses before the library sees it: matrices that do not lie as the descriptor says (CPU only; the
library's call is replaced by one that counts)."""
import pytest
import torch

import paper_2511_10054_amd as bm
from paper_2511_10054_amd import binding

ROWS, KD, N = 6, 64, 96


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Library:
        @staticmethod
        def bm_add_adapters(*args):
            made.append(args)
            return 0

    monkeypatch.setattr(binding, "load_library", lambda: Library)
    return made


def add(x, base, y, rows=ROWS, **strides):
    desc = bm.AdapterDesc(rows=rows, Kd=KD, N=N, n=2, rank=8, dtype=bm.BM_BF16, y_dtype=bm.BM_F32, **strides)
    a, b = torch.zeros((2, 8, KD), dtype=torch.bfloat16), torch.zeros((2, N, 8), dtype=torch.bfloat16)
    bm.bm_add_adapters(desc, x, torch.zeros(rows, dtype=torch.int32), a, b, None, None, base, y, torch.zeros(256, dtype=torch.uint8), stream=0)


def arrays(width=0, rows=ROWS):
    return dict(x=torch.zeros((rows, KD), dtype=torch.bfloat16), base=torch.zeros((rows, N + width)), y=torch.zeros((rows, N + width)))


@pytest.mark.parametrize("which", ["x", "base", "y"])
@pytest.mark.parametrize("change", [
    lambda t: t[:, :-1].contiguous(), lambda t: t[:, :-1],                                   # narrower: rows would be read past the last one's end
    lambda t: torch.cat([t, t], 1), lambda t: torch.cat([t, t], 1)[:, : t.shape[1]],         # wider, and columns of a wider matrix without a stride
    lambda t: t[:-1], lambda t: t.flatten()[:-1], lambda t: t.t().contiguous(), lambda t: t.t().contiguous().t(),
    lambda t: t.view(2, 3, -1)[:, :, :-1].contiguous(), lambda t: t.view(2, 3, -1)[:, :2].contiguous(),
], ids=["narrow", "narrow-view", "wide", "wide-view", "short", "short-flat", "turned", "turned-view", "narrow-3d", "short-3d"])
def test_matrices_that_are_not_the_descriptors(calls, which, change):
    t = arrays()
    t[which] = change(t[which])
    with pytest.raises(AssertionError):
        add(**t)
    assert not calls


@pytest.mark.parametrize("which", ["x", "base", "y"])
def test_strides_that_are_not_the_descriptors(calls, which):
    width = KD if which == "x" else N
    for rows, stride, named in ((ROWS, width + 8, width + 16), (ROWS, width + 8, width), (ROWS - 1, width + 8, width + 8), (ROWS, width, width + 8)):
        t = arrays()
        t[which] = torch.zeros((rows, stride), dtype=t[which].dtype)[:, :width]
        with pytest.raises(AssertionError):
            add(**t, **{which + "_stride": named})
    assert not calls


def test_matrices_that_are(calls):
    add(**arrays())
    add(**arrays(rows=ROWS + 2))                                                             # more rows than the call takes
    add(**{k: v.view(2, 3, -1) for k, v in arrays().items()})                                # tokens of a padded batch
    add(**{k: v.flatten() for k, v in arrays().items()})
    add(**arrays(rows=1), rows=1, x_stride=KD + 8, base_stride=N + 8, y_stride=N + 8)        # (of one row the stride does not matter)
    wide = {k: torch.zeros((ROWS, v.shape[1] + 8), dtype=v.dtype)[:, : v.shape[1]] for k, v in arrays().items()}
    add(**wide, x_stride=KD + 8, base_stride=N + 8, y_stride=N + 8)
    add(**arrays(), x_stride=KD, base_stride=N, y_stride=N)
    add(None, None, None, rows=0)                                                            # (the library's to refuse)
    assert len(calls) == 8
