"""The entry points beside the layer take tensors of one device: a tensor on another one is refused by name, before anything reads its pointer
(no GPU: the tensors are fake ones, which have a device and no memory)."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2403_07221_amd import binding as B


def fakes(device, *shapes):
    return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in shapes]


def refused(f, args, i, name):
    """Argument i on a second device."""
    with FakeTensorMode():
        args = list(args)
        args[i] = torch.empty(args[i].shape, dtype=args[i].dtype, device="cuda:1")
    with pytest.raises(ValueError, match=f"{name} lives on cuda:1, the call's device is cuda:0"):
        f(*args)


@pytest.fixture
def step():
    i32, f32, f8 = torch.int32, torch.float32, torch.float8_e4m3fn
    with FakeTensorMode():
        return fakes("cuda:0", ((3, 4, 64), f32), ((3, 2, 64), f32), ((3, 2, 64), f32), ((64,), f32), ((64,), f32), ((9, 64), f32), ((3,), i32),
                     ((3,), i32), ((7, 2, 16, 64), f8), ((7, 2, 64, 16), f8), ((7, 2), f32), ((7, 2), f32), ((3, 4, 64), f32))


# (the first argument is the call's device; data pointers of those before the one in question are asked for, which fake tensors warn of)
@pytest.mark.filterwarnings("ignore")
def test_tensors_on_another_device(step):
    q, k, v, qw, kw, angles, positions, slots, kc, vc, ks, vs, out = step
    for i, name in ((1, "k"), (2, "q_weight"), (3, "k_weight"), (4, "angles"), (5, "positions"), (6, "q_out"), (7, "k_out")):
        refused(B.lookupffn_rotate, (q, k, qw, kw, angles, positions, out, v), i, name)
    names = ("q", "k", "v", "q_weight", "k_weight", "angles", "positions", "slots", "k_cache", "v_cache", "k_scale", "v_scale", "q_out")
    for i, name in enumerate(names[1:], 1):
        refused(B.lookupffn_rotate_append, (q, k, v, qw, kw, angles, positions, slots, kc, vc, ks, vs, out), i, name)
    with FakeTensorMode():
        table, starts, lengths = fakes("cuda:0", ((2, 5), torch.int32), ((3,), torch.int32), ((2,), torch.int32))
        ws = torch.empty(4096, dtype=torch.uint8, device="cuda:1")
        counts = fakes("cuda:0", ((2,), torch.int32), ((2,), torch.int32), ((9,), torch.int32))
    names = ("q", "k_cache", "v_cache", "k_scale", "v_scale", "table", "starts", "lengths", "y")
    for i, name in enumerate(names[1:], 1):
        refused(B.lookupffn_attend, (q, kc, vc, ks, vs, table, starts, lengths, out), i, name)
    with pytest.raises(ValueError, match="workspace lives on cuda:1"):
        B.lookupffn_attend(q, kc, vc, ks, vs, table, starts, lengths, out, workspace=ws)
    for i, name in ((1, "fresh"), (2, "free"), (3, "table")):
        refused(lambda *a: B.lookupffn_plan_cache(*a, 5, 16), (*counts, table), i, name)
    for i, name in enumerate(("starts", "lengths", "slots", "positions", "counts")):
        shapes = ((3,), (2,), (5,), (5,), (2,))
        with FakeTensorMode():
            outs = [torch.empty(s, dtype=torch.int32, device="cuda:1" if j == i else "cuda:0") for j, s in enumerate(shapes)]
        with pytest.raises(ValueError, match=f"{name} lives on cuda:1"):
            B.lookupffn_plan_cache(*counts, table, 5, 16, *outs)
