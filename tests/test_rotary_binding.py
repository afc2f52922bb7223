"""What libra_append_attn_rotary's binding refuses of its block table, workspace and outputs."""
import pytest
import torch

from paper_2606_03077_amd import libra

ROWS, BATCH, STRIDE, HQ, HKV = 5, 2, 4, 4, 2


def arguments(device):
    """By name, in the call's order from positions on."""
    z = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=device)
    return dict(positions=z(ROWS, torch.int32), q=z((ROWS, HQ, 128), torch.bfloat16),
                k_new=z((ROWS, HKV, 128), torch.bfloat16), v_new=z((ROWS, HKV, 128), torch.bfloat16),
                block_table=z((BATCH, STRIDE), torch.int32), bt_stride=STRIDE, batch=BATCH,
                num_q_heads=HQ, scale=0.1, workspace=z(4096, torch.uint8),
                out=z((ROWS, HQ, 128), torch.bfloat16), lse=z((ROWS, HQ), torch.float32))


BAD = {  # argument: what is wrong about it -> that instead
    "block_table": [lambda t: t.long(), lambda t: t[:1], lambda t: t[:, :3].contiguous(), lambda t: t.t(),
                    lambda t: t.float()],
    "workspace": [lambda t: t[::2]],
    "out": [lambda t: t[:ROWS - 1], lambda t: t[:, :3].contiguous(), lambda t: t.float(), lambda t: t.half(),
            lambda t: t[:, :, :64].contiguous(), lambda t: t.transpose(0, 1)],
    "lse": [lambda t: t[:ROWS - 1], lambda t: t.double(), lambda t: t.bfloat16(), lambda t: t.t()],
}


@pytest.fixture()
def calls(monkeypatch):
    """The calls that reach the library."""
    made = []

    class Library:
        def libra_append_attn_rotary(self, *args):
            made.append(args)
            return 0

    monkeypatch.setattr(libra, "load", Library)
    return made


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_refused_arguments(calls, monkeypatch, device):
    """On the CPU, its tensors are those of the current device here (their index is -1)."""
    if device == "cpu":
        monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
        monkeypatch.setattr(libra, "_stream", lambda *a: None)
    a = arguments(device)
    libra.libra_append_attn_rotary(1, 2, 3, **a)
    libra.libra_append_attn_rotary(1, 2, 3, **dict(a, lse=None, out=a["out"].view(torch.int16)))
    larger = torch.zeros((ROWS + 3, HQ, 128), dtype=torch.bfloat16, device=device)
    libra.libra_append_attn_rotary(1, 2, 3, **dict(a, out=larger, block_table=a["block_table"].view(-1)))
    libra.libra_append_attn_rotary(1, 2, 3, **dict(a, block_table=a["block_table"].data_ptr()))
    assert len(calls) == 4
    assert calls[0][12] == calls[3][12] == a["block_table"].data_ptr()
    assert calls[0][-3] == a["out"].data_ptr() and calls[0][-2] == a["lse"].data_ptr()
    for name, wrong in BAD.items():
        for i, change in enumerate(wrong):
            with pytest.raises(ValueError, match=name):
                libra.libra_append_attn_rotary(1, 2, 3, **dict(a, **{name: change(a[name])}))
    assert len(calls) == 4


@pytest.mark.parametrize("name", list(BAD))
def test_tensors_of_another_device(calls, monkeypatch, name):
    """One argument at a time lies elsewhere."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(libra, "_stream", lambda *a: None)
    a = arguments("cpu")

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1

    a[name] = a[name].as_subclass(Elsewhere)
    with pytest.raises(ValueError, match=f"{name}.*current device"):
        libra.libra_append_attn_rotary(1, 2, 3, **a)
    assert not calls
