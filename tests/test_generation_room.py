"""A generation with drafts in a session whose pages or whose model's positions end
before the drafts do is refused before anything is computed."""
import os

import pytest
import torch

import paper_2606_02955_amd as fd
from workloads import cached_generation as cg

CFG = cg.Config(layers=1, hidden=64, heads=1, kv_heads=1, head_dim=64, vocab=50)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(fd.LIB_PATH) or not os.path.exists(fd.BINDING_PATH):
        from paper_2606_02955_amd import build
        build.build()


def _session(lens, gen, room, positions=4096):
    return cg.Session(cg.Model(CFG, positions, device="cpu"), lens, gen, room)


@pytest.mark.parametrize("lens,gen,room,width,depth", [
    ([64], 64, 0, 3, 4), ([64, 1], 64, 0, 3, 4), ([1, 60], 64, 3, 1, 20), ([32, 32], 32, 0, 63, 1)])
def test_no_room_for_the_drafts(lens, gen, room, width, depth):
    s = _session(lens, gen, room)
    with pytest.raises(ValueError, match="room"):
        s.generate_drafted(torch.zeros(len(lens), dtype=torch.int64), width, depth)
    assert s.done.tolist() == lens


def test_no_positions_for_the_drafts():
    # (generations without drafts need 128 of them)
    s = _session([64, 9], 64, 64, positions=130)
    with pytest.raises(ValueError, match="room"):
        s.generate_drafted(torch.zeros(2, dtype=torch.int64))


@pytest.mark.parametrize("done,fits", [(115, True), (116, False), (128, False)])
def test_a_step_behind_the_last_that_fits(done, fits):
    s = _session([64, 1], 64, 0)          # two pages a sequence
    s.done = torch.tensor([5, done])
    ids, parents = torch.zeros((2, 13), dtype=torch.int32), torch.zeros(13, dtype=torch.int32)
    # the call that fits goes on to the kernels, which want tensors on a GPU
    for call in (lambda: s.tree_hidden(ids, parents), lambda: s.drafted_step(torch.zeros(2, dtype=torch.int64), 3, 4, 0.0)):
        with pytest.raises(ValueError, match="GPU" if fits else "room"):
            call()


@pytest.mark.parametrize("lens,gen,room,width,depth", [([52], 64, 0, 3, 4), ([64], 32, 26, 3, 4), ([129, 1], 32, 64, 3, 4)])
def test_room_enough(lens, gen, room, width, depth):
    s = _session(lens, gen, room)
    with pytest.raises(ValueError, match="GPU"):
        s.generate_drafted(torch.zeros(len(lens), dtype=torch.int64), width, depth)
