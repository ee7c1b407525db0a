"""The cache in 4 bits on the host: the reference of its format against worked values, the refusals of its
entry points (nothing here reaches the GPU), and the native structures."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2406_11016_amd import binding, paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError
from paper_2406_11016_amd.paged_cache import AppendDesc, AttendDesc, PagedCache, ReadDesc
from tests import cache4_util as C4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, DTYPE, PARAM, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.fail("libspec_verify.so not built; run __graft_entry__.build()")
    return paged_cache.load_library()


def _block(*values, dtype=torch.float16, size=32):
    x = torch.zeros(size, dtype=torch.float32)
    x[:len(values)] = torch.tensor(values)
    return x.to(dtype)


def test_rounding_of_worked_blocks():
    # the largest magnitude comes into 3.5 .. 7
    for most, e in ((3.5, 0), (6.0, 0), (6.99, 0), (7.0, 1), (8.0, 1), (13.9, 1), (14.0, 2), (3.49, -1), (1.75, -1), (1.0, -2), (0.875, -2),
                    (0.874, -3), (65504.0, 14)):
        _, s = C4.quantise(_block(most))
        assert int(s[0]) == 127 + e, most
    # nearest, even code in the middle, 6 beyond, signs kept
    x = [6.0, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 3.49, 5.0, 5.01, -0.25, -0.75, -5.0, -6.9, 6.9]
    c, _ = C4.quantise(_block(*x))
    got = C4.values(c, np.array([127]))[:len(x)]
    assert got.tolist() == [6, 0, 0.5, 1, 0.5, 1, 1.5, 2, 2, 3, 4, 3, 4, 6, 0, -1, -4, -6, 6]
    assert c[14] == 8
    # bounds of the scale: zeros, subnormals
    for t, least in C4.LEAST.items():
        assert int(C4.quantise(_block(0.0, dtype=t))[1][0]) == least + 127
    c, s = C4.quantise(torch.tensor([2.0 ** -24, 3 * 2.0 ** -24] + [0.0] * 30, dtype=torch.float16))
    assert int(s[0]) == 104 and C4.values(c, s)[:2].tolist() == [2.0 ** -24, 3 * 2.0 ** -24]
    # not finite: the block is NaN, its neighbour is not
    for bad in (float("inf"), float("-inf"), float("nan")):
        x = torch.ones(80, dtype=torch.bfloat16)
        x[70] = bad
        v = C4.values(*C4.quantise(x))
        assert np.isnan(v[64:]).all() and (v[:64] == 1).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_held_value_is_of_the_type_and_within_a_sixth_of_the_largest(dtype):
    """Off by at most half the distance of two numbers or by what is beyond 6, relative to the block's largest magnitude,
    which is the value itself or more: 5 goes to 4, a fifth; 3.5 to 4 and 2.5 to 2 of 3.5 or more, a seventh; less than 7
    to 6, a seventh.  (Where the scale's bound acts, a quarter of it: 0.25 goes to 0.)"""
    x = torch.randn(200, 96, generator=torch.Generator().manual_seed(1)) * torch.logspace(-3, 3, 200)[:, None]
    x = x.to(dtype)
    v = C4.values(*C4.quantise(x))
    assert np.array_equal(torch.from_numpy(v).to(dtype).double().numpy(), v)
    blocks = np.abs(x.double().numpy()).reshape(200, 3, 32)
    off = np.abs(v - x.double().numpy()).reshape(200, 3, 32)
    assert (off <= np.maximum(blocks.max(-1, keepdims=True) / 5, 2.0 ** C4.LEAST[dtype] / 4)).all()
    # and what is held is held exactly
    again = C4.quantise(torch.from_numpy(v).to(dtype))
    assert np.array_equal(C4.values(*again), v)


def test_layout():
    x = torch.randn(2, 3, 16, 80, generator=torch.Generator().manual_seed(2)).to(torch.float16)
    p = C4.pack(x)
    assert p.shape == (2, 3, 16 * paged_cache.row_bytes4(80)) and paged_cache.row_bytes4(80) == C4.row_bytes(80) == 43
    codes, scales = C4.quantise(x)
    assert int(p[1, 2, 5 * 40 + 7]) == codes[1, 2, 5, 14] | codes[1, 2, 5, 15] << 4
    assert int(p[1, 2, 16 * 40 + 5 * 3 + 2]) == scales[1, 2, 5, 2]
    assert np.array_equal(C4.unpack(p, 16, 80, "f16").double().numpy(), C4.values(codes, scales))


def test_read_structure_is_the_headers(tmp_path):
    lines = ['printf("%zu\\n", sizeof(sv_cache_read_desc_t));']
    lines += [f'printf("%zu\\n", offsetof(sv_cache_read_desc_t, {f[0]}));' for f in ReadDesc._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "spec_cache.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\nreturn 0; }\n")
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(ReadDesc)] + [getattr(ReadDesc, f[0]).offset for f in ReadDesc._fields_]


ROW = 64 + 4  # bytes of a token and head at head_dim 128


def _rows_call(f, cls, **kw):
    i3 = ctypes.c_int64 * 3
    d = dict(k=0x1000, v=0x2000, k_stride=(512, 256, 128), v_stride=(512, 256, 128), k_cache=0x3000, v_cache=0x4000,
             page_stride=2 * 16 * ROW, slots=0x5000, dtype=binding.SV_F16, batch=2, max_new=3, kv_heads=2, head_dim=128,
             num_pages=8, page_size=16)
    d.update(kw)
    d["k_stride"], d["v_stride"] = i3(*d["k_stride"]), i3(*d["v_stride"])
    return f(ctypes.byref(cls(**d)), None)


@pytest.mark.parametrize("name", ["append4", "read4"])
def test_bad_append_and_read_arguments(lib, name):
    f, cls = getattr(lib, "spec_cache_" + name), AppendDesc if name == "append4" else ReadDesc
    assert f(None, None) == NULL
    for field in ("k", "v", "k_cache", "v_cache", "slots"):
        assert _rows_call(f, cls, **{field: None}) == NULL
    for code in (binding.SV_F32, 3, -1):
        assert _rows_call(f, cls, dtype=code) == DTYPE
    for kw in (dict(batch=0), dict(batch=4097), dict(max_new=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=12),
               dict(num_pages=0), dict(page_size=8), dict(page_size=48), dict(num_pages=1 << 28), dict(max_new=1 << 30),
               dict(max_new=1 << 28, kv_heads=64, page_stride=1 << 20)):
        assert _rows_call(f, cls, **kw) == SHAPE, kw
    for kw in (dict(page_stride=2 * 16 * ROW - 16), dict(page_stride=2 * 16 * ROW + 8), dict(k=0x1004), dict(v=0x2008),
               dict(k_cache=0x3008), dict(v_cache=0x4002), dict(k_stride=(512, 260, 128)), dict(v_stride=(-8, 256, 128))):
        assert _rows_call(f, cls, **kw) == PARAM, kw
    if name == "read4":   # rows that lie on one another would be written by several threads
        for i in range(3):
            strides = [768, 256, 128]
            strides[i] = 0
            assert _rows_call(f, cls, k_stride=tuple(strides)) == PARAM
            assert _rows_call(f, cls, v_stride=tuple(strides)) == PARAM


def _attend(lib, **kw):
    i3 = ctypes.c_int64 * 3
    d = dict(q=0x1000, out=0x2000, q_stride=(1024, 512, 128), out_stride=(1024, 512, 128), k_cache=0x3000, v_cache=0x4000,
             page_stride=2 * 16 * ROW, block_table=0x5000, lengths=0x6000, counts=None, prefix_table=None, prefix_len=0,
             dtype=binding.SV_BF16, batch=2, max_new=3, q_heads=4, kv_heads=2, head_dim=128, max_pages=4, num_pages=8,
             page_size=16, scale=0.1, workspace=0x7000, workspace_bytes=1 << 40)
    d.update(kw)
    d["q_stride"], d["out_stride"] = i3(*d["q_stride"]), i3(*d["out_stride"])
    return lib.spec_cache_attend4(ctypes.byref(AttendDesc(**d)), None)


def test_bad_attend_arguments(lib):
    assert lib.spec_cache_attend4(None, None) == NULL
    for f in ("q", "out", "k_cache", "v_cache", "block_table", "lengths", "workspace"):
        assert _attend(lib, **{f: None}) == NULL
    assert _attend(lib, prefix_len=3) == NULL
    assert _attend(lib, dtype=binding.SV_F32) == DTYPE
    for kw in (dict(q_heads=3), dict(head_dim=120), dict(batch=0), dict(max_new=0), dict(max_pages=0),
               dict(prefix_len=-1, prefix_table=0x100)):
        assert _attend(lib, **kw) == SHAPE, kw
    assert _attend(lib, batch=1024, q_heads=65536, kv_heads=65536, max_pages=1 << 20, page_stride=65536 * 16 * ROW) == SHAPE
    for kw in (dict(scale=0.0), dict(scale=float("nan")), dict(q=0x1002), dict(out_stride=(1024, 512, 4)),
               dict(out_stride=(1024, 0, 128)), dict(page_stride=2 * 16 * ROW + 8), dict(page_stride=2 * 16 * ROW - 16),
               dict(k_cache=0x3008)):
        assert _attend(lib, **kw) == PARAM, kw
    need = lib.spec_cache_attend4_workspace_bytes(2, 3, 4, 2, 128)
    assert need > 0 and _attend(lib, workspace_bytes=need - 1) == WORKSPACE and _attend(lib, workspace=0x7008) == WORKSPACE
    assert lib.spec_cache_attend4_workspace_bytes(2, 3, 5, 2, 128) == 0
    assert lib.spec_cache_attend4_workspace_bytes(2, 3, 4, 2, 72) == 0


def test_host_tensors_and_other_types_are_refused():
    x = torch.zeros(2, 3, 2, 64, dtype=torch.float16)
    c = torch.zeros(4, 2, 16 * 34, dtype=torch.uint8)
    i = torch.zeros(2, 3, dtype=torch.int32)
    for call in (lambda: paged_cache.append4(x, x, c, c, i), lambda: paged_cache.read4(c, c, i, 64, torch.float16),
                 lambda: paged_cache.read4(c, c, i), lambda: paged_cache.read4(c, c, i, 64, torch.float32),
                 lambda: paged_cache.append4(x.float(), x.float(), c, c, i),
                 lambda: paged_cache.attend4(x.float(), c, c, i, i[:, 0].contiguous()),
                 lambda: paged_cache.attend4(x, c, c, i, i[:, 0].contiguous()),
                 lambda: paged_cache.new_attend4_workspace(2, 3, 5, 2, 128, "cpu")):
        with pytest.raises(SpecVerifyError):
            call()


def test_storage_arguments():
    cache = PagedCache.__new__(PagedCache)
    cache.num_pages, cache.page_size, cache.device = 5, 16, torch.device("cpu")
    k, v = cache.new_storage(3, 80, torch.float16, bits=4)
    assert k.shape == v.shape == (5, 3, 16 * 43) and k.dtype == torch.uint8
    assert cache.new_storage(3, 80, torch.float16)[0].shape == (5, 3, 16, 80)
    assert cache._described(k, 80) and not cache._described(cache.new_storage(3, 80, torch.float16)[0], 80)
    for bad in (lambda: cache.new_storage(3, 80, torch.float16, bits=8), lambda: cache.new_storage(3, 80, torch.uint8, bits=4),
                lambda: cache.new_storage(3, 84, torch.float16, bits=4), lambda: cache._described(k, 64),
                lambda: cache._described(k[:4], 80), lambda: cache._described(k[:, :, None], 80)):
        with pytest.raises(SpecVerifyError):
            bad()
