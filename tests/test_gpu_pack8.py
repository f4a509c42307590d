"""8-bit checkpoints against their oracle: every step is exact, so codes, scales and what is read back are equal."""
import numpy as np
import pytest
import torch

from oracle import pack8 as K
from paper_2608_21308_b200 import binding as E
from paper_2608_21308_b200 import inputs

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def through(x, io):
    p = E.make_pack_params(*x.shape, E.E2TTT_F32 if io == "f32" else E.E2TTT_BF16)
    codes = torch.full(x.shape, 77, dtype=torch.int8, device="cuda")
    scales = torch.full((x.shape[0], -(-x.shape[1] // 32)), 77, dtype=torch.uint8, device="cuda")
    back = torch.full_like(x, 7.0)
    E.e2ttt_pack8(p, x, codes, scales)
    E.e2ttt_unpack8(p, codes, scales, back)
    return codes, scales, back


def check(a, io, x=None):
    x = torch.tensor(a, device="cuda").to(DT[io]) if x is None else x
    codes, scales, back = through(x, io)
    rc, rs = K.pack(a)
    assert np.array_equal(scales.cpu().numpy(), rs)
    assert np.array_equal(codes.cpu().numpy(), rc)
    assert np.array_equal(back.double().cpu().numpy(), K.unpack(rc, rs), equal_nan=True)


def values(rows, cols, io, seed=0):
    rng = np.random.default_rng(seed)
    a = (np.exp(2 * rng.standard_normal((rows, 1))) * rng.standard_normal((rows, cols))).astype(np.float32)
    return inputs.round_bf16(a) if io == "bf16" else a


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 64), (300, 8), (4, 777), (9, 40), (1, 5000), (130, 96), (2, 36), (3, 34), (40, 2048)])
def test_equal_to_the_oracle(io, rows, cols):
    check(values(rows, cols, io), io)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_tensors_at_any_element(io, shift):
    a = values(11, 96, io, 1)
    x = torch.zeros(a.size + shift, device="cuda", dtype=DT[io])[shift:].view(a.shape)
    x.copy_(torch.tensor(a))
    check(a, io, x)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_ends_of_the_range_zeros_ties_and_values_that_are_not_finite(io):
    top = float(torch.finfo(DT[io]).max)
    rows = [np.zeros(32), np.full(32, top), np.r_[top, -top, np.zeros(30)], np.full(32, 2.0 ** -126), np.r_[2.0 ** -133, np.zeros(31)], np.r_[127.0, 0.5 + np.arange(31)],
            np.r_[127.0 / 64, np.linspace(-1, 1, 31)], np.r_[1.9921875, np.linspace(-1, 1, 31)], np.r_[np.nan, np.ones(31)], np.r_[np.ones(31), -np.inf], np.r_[np.inf, np.nan, np.ones(30)],
            np.r_[2.0 ** 121 * 127, -(2.0 ** 120)] .repeat(16), -np.arange(32.0)]
    if io == "f32":
        rows += [np.r_[1e-40, 3e-45, np.ones(30) * 1e-39], np.r_[np.nextafter(np.float32(127), np.float32(200)), np.arange(31)]]
    a = np.array(rows, dtype=np.float32)
    a = inputs.round_bf16(a) if io == "bf16" else a
    a[8:11] = np.array(rows[8:11], dtype=np.float32)
    check(a, io)
    check(np.ascontiguousarray(a.reshape(1, -1)), io)
    check(np.ascontiguousarray(a[:, :29]), io)


def test_every_code_and_scale_is_read_back():
    codes = torch.arange(-128, 128, device="cuda").to(torch.int8).repeat(256, 1)
    scales = torch.arange(256, device="cuda").to(torch.uint8)[:, None].repeat(1, 8)
    for io in ("f32", "bf16"):
        back = torch.empty(256, 256, device="cuda", dtype=DT[io])
        E.e2ttt_unpack8(E.make_pack_params(256, 256, E.E2TTT_F32 if io == "f32" else E.E2TTT_BF16), codes, scales, back)
        want = (codes.double() * torch.exp2(scales.double()[:, :1] - 127)).float().double()  # -128 2^121 = -2^128 is rounded to -inf
        got = back.double()
        assert bool(torch.isnan(got[255]).all())
        assert torch.equal(got[1:249], want[1:249])  # the bytes that are ever written


def test_more_than_two_to_the_31_elements_and_a_captured_call():
    rows, cols = (1 << 20) + 3, 2080
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    a = values(3, cols, "bf16", 2)
    x[-3:].copy_(torch.tensor(a))
    p = E.make_pack_params(rows, cols, E.E2TTT_BF16)
    codes = torch.empty(x.shape, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, cols // 32, dtype=torch.uint8, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        E.e2ttt_pack8(p, x, codes, scales)
    graph.replay()
    torch.cuda.synchronize()
    rc, rs = K.pack(a)
    assert np.array_equal(codes[-3:].cpu().numpy(), rc) and np.array_equal(scales[-3:].cpu().numpy(), rs)
    assert not bool(codes[:-3].any()) and bool((scales[:-3] == 1).all())
    E.e2ttt_unpack8(p, codes, scales, x.fill_(7.0))
    assert np.array_equal(x[-3:].double().cpu().numpy(), K.unpack(rc, rs)) and not bool(x[:-3].any())
