"""Memory bins and the envelope rule of the forecasting side (no GPU)."""
import torch

from paper_2509_19086_b200 import forecast


def test_bins_cover_every_value_from_above():
    bins = forecast.MemoryBins(256)
    mem = torch.tensor([1, 63, 64, 65, 4096, 4097, 81919, 81920])
    tok = bins.tokens(mem)
    assert (tok >= 0).all() and (tok < 256).all() and (tok[1:] >= tok[:-1]).all()
    assert (bins.upper_MiB(tok) >= mem).all()
    assert (bins.edges[(tok[2:] - 1).clamp(min=0)] < mem[2:]).logical_or(tok[2:] == 0).all()
    assert bins.upper_MiB(torch.tensor([255])).item() == 81920


def test_envelope_rule():
    lp = torch.log(torch.tensor([[0.5, 0.3, 0.15, 0.05], [0.4, 0.2, 0.1, 0.1], [1.0, 0.0, 0.0, 0.0]]))
    ids = torch.tensor([[7, 2, 9, 1], [3, 4, 5, 6], [8, 0, 1, 2]])
    assert forecast.envelope(lp, ids, 0.1, 64).tolist() == [9, 63, 8]      # second row: its alternatives hold 0.8 only
    assert forecast.envelope(lp, ids, 0.25, 64).tolist() == [7, 6, 8]      # 0.4 + 0.2 + 0.1 is short of 0.75
    assert forecast.envelope(lp, ids, 0.6, 64).tolist() == [7, 3, 8]
