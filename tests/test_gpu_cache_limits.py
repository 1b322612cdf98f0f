"""Moves, plans and paths at the largest numbers that their entry points take."""
import pytest
import torch

from beam_util import accepted_path

pytestmark = pytest.mark.gpu


def test_path_of_the_greatest_depth(gpu_lib):
    """Rows of 2^31 - 1 entries, of which all but the first few are padding."""
    N, width = 65, (1 << 31) - 1
    i32 = dict(dtype=torch.int32, device="cuda")
    parent = torch.arange(-1, N - 1, **i32).view(1, N)
    token = torch.arange(N, **i32).view(1, N) % 7
    tokens = torch.zeros((1, width), **i32)
    tokens[0, :20] = token[0, 1:21]
    print("path of", width, "entries", flush=True)
    path, st = gpu_lib.resispec_accepted_path(parent, token, tokens, torch.tensor([20], **i32))
    torch.cuda.synchronize()
    assert st.tolist() == [0]
    way = accepted_path(parent[0].tolist(), token[0].tolist(), tokens[0, :21].tolist(), 20)
    assert path[0, :21].tolist() == way
    for i in range(21, width, 1 << 28):
        part = path[0, i:i + (1 << 28)]
        assert int(part.max()) == int(part.min()) == -1, i
