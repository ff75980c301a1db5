"""What the serving loop refuses, without a GPU."""
import pytest
import torch

import paper_2410_18248_amd as P
from paper_2410_18248_amd.engine import LiveEngine


class _Recorder:
    def __init__(self):
        self.calls = []

    def batch_tables(self, *args):
        self.calls.append(args)


def _engine(row):
    eng = object.__new__(LiveEngine)
    eng.cfg = P.LampsConfig(1, 4, 2, 64, 16, 8, row, 4, P.LAMPS_BF16)
    eng.dev, eng.lam = torch.device("cpu"), _Recorder()
    eng.blocks = {0: [3], 7: [0, 1, 2]}
    return eng


def test_a_context_beyond_the_table_row_is_an_error():
    """The table call leaves such a request out and goes on: the loop must not."""
    for cached, new in ((30, 3), (0, 33), (32, 1)):
        eng = _engine(2)
        with pytest.raises(ValueError, match="request 7"):
            eng._batch([0, 7], [4, cached], [1, new])
        assert not eng.lam.calls
    for row, cached, new in ((2, 30, 2), (3, 30, 18)):
        eng = _engine(row)
        eng._batch([0, 7], [4, cached], [1, new])
        n, total, _, _, ids, n_ids = eng.lam.calls[0][:6]
        assert (n, total) == (2, 1 + new) and ids.tolist() == [3] + eng.blocks[7][:row] and n_ids == 1 + row
