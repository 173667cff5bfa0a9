"""Calls of the batch plan and of the 8-bit K/V cache that are refused (CPU): buffers that overlap, shapes and numbers that
the C structures would hold as others.  The pointers of the refused calls are never followed."""
import pytest
import torch

from paper_2605_30218_amd import mg

ARG = -1
NAMES = ("ctx_len", "n_new", "free_pages", "n_free", "page_table", "cu_new", "lens", "admitted", "positions", "rows", "slots",
         "n_left")


def plan_status(B=300, maxp=8, most=500, **at):
    """The status of a plan whose buffers stand 1 MiB apart, but for those whose addresses are given."""
    p = {n: (i + 1) << 20 for i, n in enumerate(NAMES)} | at
    return mg.load().mg_batch_plan(B, maxp, p["ctx_len"], p["n_new"], p["free_pages"], p["n_free"], most, *[p[n] for n in NAMES[4:]],
                                   None)


@pytest.mark.parametrize("name,out", [(i, o) for i in NAMES[:5] for o in NAMES[4:] if i != o])
def test_plan_outputs_on_its_inputs_are_refused(name, out):
    """Blocks of the launch read the inputs while others write: the same buffer, its last value, the value before it."""
    at = (NAMES.index(name) + 1) << 20
    values = {"ctx_len": 300, "n_new": 300, "n_free": 1, "free_pages": 1, "page_table": 300 * 8}[name]
    length = {"page_table": 300 * 8, "cu_new": 301, "lens": 300, "admitted": 300, "n_left": 1}.get(out, 500)
    for shift in (0, 4 * (values - 1), -4 * (length - 1)):
        assert plan_status(**{out: at + shift}) == ARG, shift


def cpu_call(hd=64, width=None, call=mg.kv8_attention, **kw):
    """An attention call on CPU tensors, which the binding refuses at the latest for where they are."""
    codes, scales = (torch.zeros(s, dtype=torch.uint8) for s in ((4, 2, 2, width or 16 * hd), (4, 2, 2)))
    q = torch.zeros((3, 4, hd), dtype=torch.bfloat16)
    return call(codes, scales, q, torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), **kw)


@pytest.mark.parametrize("width", [1030, 1025, 1039, 2056])
def test_codes_of_no_whole_head_are_refused(width):
    with pytest.raises(ValueError, match="codes"):
        cpu_call(width=width)


@pytest.mark.parametrize("name", ["max_new", "max_len", "window"])
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 5, 2 ** 40, -2 ** 31 - 1, -2 ** 32 + 7])
@pytest.mark.parametrize("call", [mg.kv8_attention, mg.kv8_attention_workspace_bytes])
def test_numbers_past_32_bits_are_refused(name, value, call):
    """The call's structure holds 32 bits: a window of 2^32 + 5 would be one of 5."""
    with pytest.raises(ValueError, match=name):
        cpu_call(call=call, **{name: value})


@pytest.mark.parametrize("name", ["scale", "softcap"])
@pytest.mark.parametrize("value", [1e-50, -1e-50, 1e-300])
def test_factors_that_are_zero_in_32_bits_are_refused(name, value):
    """0 stands for the default scale, and for no cap."""
    with pytest.raises(ValueError, match=name):
        cpu_call(**{name: value})


def test_a_stream_of_another_device_is_refused():
    """Its kernels would run there, on memory that need not be mapped."""
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 0

    def never(*_):
        raise AssertionError("the call was made")

    with pytest.raises(ValueError, match="stream"):
        mg._call("mg_kv8_attention", torch.device("cuda", 0), Stream(), never)
