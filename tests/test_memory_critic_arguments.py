"""What MemoryCritic refuses when it is made, on a stand-in of the library: without a GPU."""
import pytest
import torch

from paper_2107_01460_amd import memory
from memory_stand_in import StandIn


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    monkeypatch.setattr(memory, "B", StandIn)


def test_a_device_that_is_not_the_current_one(monkeypatch):
    """The kernels go to the current GPU's stream, and so does the table: parameters on another would meet them there."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for device in ("cuda:1", torch.device("cuda", 3)):
        with pytest.raises(StandIn.MarlError, match="current"):
            memory.MemoryCritic(8, width=16, heads=2, layers=1, device=device)


def test_heads_wider_than_the_attention_takes():
    with pytest.raises(StandIn.MarlError, match="128"):
        memory.MemoryCritic(8, width=258, heads=2, layers=1, device="cpu")
    memory.MemoryCritic(8, width=256, heads=2, layers=1, device="cpu")
