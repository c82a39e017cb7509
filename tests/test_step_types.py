"""The optimizer's lists of tensors and the types that a call takes: those of the same size
that mean something else are refused too."""
import pytest
import torch

from paper_2606_05484_amd import mapl

f32, bf, u8 = torch.float32, torch.bfloat16, torch.uint8


def z(dt, n=300):
    return torch.zeros(n, dtype=dt)


@pytest.mark.parametrize("dt,g_dtype", [(torch.float16, "bf16"), (torch.int16, "bf16"), (torch.int32, "f32"), (torch.float64, "f32"),
                                        (bf, "f32"), (f32, "bf16")])
def test_the_norm_refuses_gradients_of_another_type(dt, g_dtype):
    with pytest.raises(ValueError, match="type"):
        mapl.grad_norm(mapl.optim_params([z(dt)]), None, None, g_dtype=g_dtype, stream=0)


@pytest.mark.parametrize("name,dt", [("g", torch.float16), ("g", torch.int16), ("p", torch.int32), ("m", torch.int32), ("v", torch.int32), ("p16", torch.float16),
                                     ("p16", torch.int16), ("e", torch.int32)])
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_the_step_refuses_arrays_of_another_type(name, dt, states):
    state = u8 if states == "8bit" else f32
    kinds = dict(g=bf, p=f32, m=state, v=state, e=u8, p16=bf)
    kinds[name] = dt
    a = mapl.optim_params(**{k: [z(t)] for k, t in kinds.items()})
    with pytest.raises(ValueError, match="type"):
        mapl.adamw_step(mapl.adamw_desc(1e-3, g_dtype="bf16", states=states, step=1), a, stream=0)


def test_conversions_refuse_values_of_another_type():
    packed = mapl.optim_params([z(f32)], m=[z(u8)], v=[z(u8)], e=[z(u8)])
    for m, v in ((torch.int32, f32), (f32, torch.int32)):
        values = mapl.optim_params([z(f32)], m=[z(m)], v=[z(v)])
        for call in (lambda: mapl.adamw_unpack(packed, values, stream=0), lambda: mapl.adamw_pack(values, packed, stream=0)):
            with pytest.raises(ValueError, match="type"):
                call()


def test_one_kind_has_one_type():
    for x in ([z(bf), z(torch.float16)], [z(f32), z(f32), z(torch.int32)]):
        with pytest.raises(ValueError, match="type"):
            mapl.optim_params(x)


def test_codes_are_bytes_whatever_their_type_is_called():
    for dt in (u8, torch.int8, torch.float8_e4m3fn):
        a = mapl.optim_params([z(f32)], [z(f32)], [z(dt)], [z(dt)], [z(u8)])
        a.need(("g", "f32"), ("p", "f32"), ("m", "u8"), ("v", "u8"), ("e", "u8"), ("p16", "bf16"))
