"""The calls of the GPU tests of large sequences take the kernels that they are for (the launchers' own rules, host code without a GPU)."""
import ctypes

import pytest
import torch

from paper_2010_15884_amd import binding as B
from paper_2010_15884_amd import sequence as S
from test_gpu_sequence_routes import SPANS, WIDE, WIDTHS

CODES = {torch.float32: B.SYS_F32, torch.float16: B.SYS_F16, torch.bfloat16: B.SYS_BF16}


def _host(name, packed):
    fn = B.lib()[name]
    fn.argtypes, fn.restype = [ctypes.c_char_p], ctypes.c_int
    return fn(packed)


def rows_a_lane(batch, length, channels, dtype, width=4):
    code = CODES[dtype]
    return _host("_ZN7sysconv23causal_conv_rows_a_laneERK19sys_causal_conv1d_t",
                 S._CONV.pack(code, code, 0, width, batch, length, channels, 0, length * channels, channels, length * channels, channels))


def spans(batch, length, channels, states, dtype, groups):
    row = [length * channels, channels]
    bc = [length * groups * states, groups * states]
    return _host("_ZN7sysconv15scan_grad_spansERK20sys_selective_scan_t",
                 S._SCAN.pack(CODES[dtype], 1, batch, length, channels, states, groups, 0, *row, *row, *row, *bc, *bc, *row))


def test_convolutions_of_many_rows():
    assert {dtype for _, _, _, dtype, _ in WIDE} == set(CODES) and WIDTHS == list(range(2, B.SYS_MAX_CAUSAL_WIDTH + 1))
    for dtype in CODES:
        assert {channels < 16 // dtype.itemsize for _, _, channels, kind, _ in WIDE if kind == dtype} == {True, False}
    for batch, length, channels, dtype, _ in WIDE:
        assert rows_a_lane(batch, length, channels, dtype) == 16
    assert rows_a_lane(5, 1021, 1001, torch.float16) == 4


def test_gradients_in_chunks_of_several_spans():
    for want, case in SPANS:
        assert spans(*case[:6]) == want
    assert {want for want, _ in SPANS} == set(range(2, 9))
    # 1, 2, 4, 8 and 16 states a lane
    assert {max(1, 1 << (-(-case[3] // 4) - 1).bit_length()) for _, case in SPANS} == {1, 2, 4, 8, 16}


@pytest.mark.parametrize("blocks,want", [(1023, 1), (1024, 2), (1535, 2), (1536, 3), (4095, 7), (4096, 8), (20000, 8)])
def test_lines_of_the_spans(blocks, want):
    assert spans(blocks, 16, 64, 16, torch.bfloat16, 1) == want


def test_lines_of_the_rows():
    for batch, length, channels, dtype in ((1, 6144, 4096, torch.bfloat16), (1, 6144, 2048, torch.float32), (3, 1 << 20, 1, torch.float16)):
        assert rows_a_lane(batch, length, channels, dtype) == 16 and rows_a_lane(batch, length - 1, channels, dtype) == 4
