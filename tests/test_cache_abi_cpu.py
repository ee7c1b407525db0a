"""The key/value cache's C ABI on the host: the library exports what
spec_cache.h declares, the binding's structures are the header's, and invalid
arguments are rejected before anything is launched (no call here reaches the
GPU).  And the library's device code, the cache's kernels among it: no
packed-fp32 instructions, no scratch memory."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2406_11016_amd import binding, paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError
from paper_2406_11016_amd.decode_loop import DecodeLoop
from paper_2406_11016_amd.paged_cache import AppendDesc, AttendDesc, PagedCache, Tables

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "spec_cache.h")
LLVM = "/opt/rocm/lib/llvm/bin"
OK, NULL, SHAPE, DTYPE, PARAM, WORKSPACE = 0, -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.fail("libspec_verify.so not built; run __graft_entry__.build()")
    return paged_cache.load_library()


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(spec_cache_\w+)\s*\(", text)))


def test_header_and_exports(lib):
    assert _declared() == sorted(paged_cache.SYMBOLS)
    out = subprocess.run(["nm", "-D", "--defined-only", binding.LIB_PATH], capture_output=True, text=True,
                         check=True).stdout
    assert sorted(re.findall(r"\bT (spec_cache_\w+)", out)) == _declared()


def test_structures_are_the_headers(tmp_path):
    """Sizes and offsets of the ctypes structures, against the C compiler's."""
    pairs = [(Tables, "sv_cache_tables_t"), (AppendDesc, "sv_cache_append_desc_t"), (AttendDesc, "sv_cache_attend_desc_t")]
    lines = []
    for cls, name in pairs:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "spec_cache.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\nreturn 0; }\n")
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for cls, _ in pairs:
        want += [ctypes.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_]
    assert got == want
    # and what the binding packs in one go
    i3 = ctypes.c_int64 * 3
    a = list(range(1, 20))
    d = AppendDesc(1, 2, i3(3, 4, 5), i3(6, 7, 8), *a[8:])
    assert bytes(d) == paged_cache._pack_append(*a)
    a = list(range(1, 29))
    a[25] = 0.75                                             # scale
    d = AttendDesc(1, 2, i3(3, 4, 5), i3(6, 7, 8), *a[8:])
    assert bytes(d) == paged_cache._pack_attend(*a)


def _tables(**kw):
    t = dict(lengths=0x1000, counts=0x2000, held=0x3000, block_table=0x4000, free_pages=0x5000, free_count=0x6000, batch=2,
             max_pages=3, num_pages=8, page_size=16)
    t.update(kw)
    return Tables(**t)


BAD_TABLES = [(NULL, {f: None}) for f in ("lengths", "counts", "held", "block_table", "free_pages", "free_count")]
BAD_TABLES += [(SHAPE, kw) for kw in (dict(batch=0), dict(batch=4097), dict(max_pages=0), dict(num_pages=0),
                                      dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(page_size=0),
                                      dict(page_size=-16), dict(num_pages=1 << 27), dict(max_pages=1 << 27),
                                      dict(batch=4096, max_pages=1 << 20))]


@pytest.mark.parametrize("want,kw", BAD_TABLES, ids=[str(b[1]) for b in BAD_TABLES])
def test_bad_tables(lib, want, kw):
    t = ctypes.byref(_tables(**kw))
    assert lib.spec_cache_init(t, 0, None) == want
    assert lib.spec_cache_plan(t, None, None, None, 4, 0, 0x7000, None, None) == want


def test_bad_plan_and_init_arguments(lib):
    t = ctypes.byref(_tables())
    assert lib.spec_cache_init(None, 0, None) == NULL
    assert lib.spec_cache_init(t, -1, None) == SHAPE and lib.spec_cache_init(t, 9, None) == SHAPE
    assert lib.spec_cache_plan(None, None, None, None, 4, 0, 0x7000, None, None) == NULL
    assert lib.spec_cache_plan(t, None, None, None, 4, 0, None, None, None) == NULL
    for n in (0, -1, 1 << 30):
        assert lib.spec_cache_plan(t, None, None, None, n, 0, 0x7000, None, None) == SHAPE
    for base in (-1, (1 << 31) - 1):
        assert lib.spec_cache_plan(t, None, None, None, 4, base, 0x7000, None, None) == PARAM


def _append(lib, **kw):
    i3 = ctypes.c_int64 * 3
    d = dict(k=0x1000, v=0x2000, k_stride=(512, 256, 128), v_stride=(512, 256, 128), k_cache=0x3000, v_cache=0x4000,
             page_stride=2 * 16 * 128, slots=0x5000, dtype=binding.SV_F16, batch=2, max_new=3, kv_heads=2, head_dim=128,
             num_pages=8, page_size=16)
    d.update(kw)
    d["k_stride"], d["v_stride"] = i3(*d["k_stride"]), i3(*d["v_stride"])
    return lib.spec_cache_append(ctypes.byref(AppendDesc(**d)), None)


def test_bad_append_arguments(lib):
    assert lib.spec_cache_append(None, None) == NULL
    for f in ("k", "v", "k_cache", "v_cache", "slots"):
        assert _append(lib, **{f: None}) == NULL
    for code in (binding.SV_F32, 3, -1):
        assert _append(lib, dtype=code) == DTYPE
    for kw in (dict(batch=0), dict(batch=4097), dict(max_new=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=12),
               dict(num_pages=0), dict(page_size=8), dict(page_size=48), dict(num_pages=1 << 28), dict(max_new=1 << 30),
               dict(max_new=1 << 28, kv_heads=64, page_stride=1 << 20)):
        assert _append(lib, **kw) == SHAPE, kw
    for kw in (dict(page_stride=2 * 16 * 128 - 8), dict(page_stride=2 * 16 * 128 + 2), dict(k=0x1004), dict(v=0x2008),
               dict(k_cache=0x3002), dict(v_cache=0x4008), dict(k_stride=(512, 260, 128)), dict(v_stride=(-8, 256, 128))):
        assert _append(lib, **kw) == PARAM, kw


def _attend(lib, **kw):
    i3 = ctypes.c_int64 * 3
    d = dict(q=0x1000, out=0x2000, q_stride=(1024, 512, 128), out_stride=(1024, 512, 128), k_cache=0x3000, v_cache=0x4000,
             page_stride=2 * 16 * 128, block_table=0x5000, lengths=0x6000, counts=None, prefix_table=None, prefix_len=0,
             dtype=binding.SV_BF16, batch=2, max_new=3, q_heads=4, kv_heads=2, head_dim=128, max_pages=4, num_pages=8,
             page_size=16, scale=0.1, workspace=0x7000, workspace_bytes=1 << 40)
    d.update(kw)
    d["q_stride"], d["out_stride"] = i3(*d["q_stride"]), i3(*d["out_stride"])
    return lib.spec_cache_attend(ctypes.byref(AttendDesc(**d)), None)


def test_bad_attend_arguments(lib):
    """A few through the ABI; the whole contract is checked on check_attend (tests/native/cache_check.cpp)."""
    assert lib.spec_cache_attend(None, None) == NULL
    for f in ("q", "out", "k_cache", "v_cache", "block_table", "lengths", "workspace"):
        assert _attend(lib, **{f: None}) == NULL
    assert _attend(lib, prefix_len=3) == NULL
    assert _attend(lib, dtype=binding.SV_F32) == DTYPE
    for kw in (dict(q_heads=3), dict(head_dim=120), dict(batch=0), dict(max_new=0), dict(max_pages=0), dict(prefix_len=-1, prefix_table=0x100)):
        assert _attend(lib, **kw) == SHAPE, kw
    # more units than 31 bits count: refused, not wrapped
    assert _attend(lib, batch=1024, q_heads=65536, kv_heads=65536, max_pages=1 << 20, page_stride=65536 * 16 * 128) == SHAPE
    for kw in (dict(scale=0.0), dict(scale=float("nan")), dict(q=0x1002), dict(out_stride=(1024, 512, 4))):
        assert _attend(lib, **kw) == PARAM, kw
    need = lib.spec_cache_attend_workspace_bytes(2, 3, 4, 2, 128)
    assert need > 0 and _attend(lib, workspace_bytes=need - 1) == WORKSPACE and _attend(lib, workspace=0x7008) == WORKSPACE
    assert lib.spec_cache_attend_workspace_bytes(2, 3, 5, 2, 128) == 0


def test_host_tensors_are_refused():
    x = torch.zeros(2, 3, 2, 64, dtype=torch.float16)
    c = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    i = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(SpecVerifyError):
        paged_cache.append(x, x, c, c, i)
    with pytest.raises(SpecVerifyError):
        paged_cache.attend(x, c, c, i, i[:, 0].contiguous())
    with pytest.raises(SpecVerifyError):
        PagedCache(2, num_pages=4, page_size=16, max_pages=2, max_new=3, device="cpu")
    with pytest.raises(SpecVerifyError):
        PagedCache(0, num_pages=4, page_size=16, max_pages=2, max_new=3)
    with pytest.raises(SpecVerifyError):
        paged_cache.new_attend_workspace(2, 3, 5, 2, 128, "cpu")


def test_loop_refuses_a_cache_that_does_not_fit():
    class Other:
        batch, max_new, device = 3, 5, torch.device("cuda", 0)
    for kw in (dict(batch=2), dict(gamma_max=5)):
        args = dict(batch=3, vocab=100, dtype="f32", gamma0=1, gamma_max=4, cache=Other(), device="cuda")
        args.update(kw)
        with pytest.raises(ValueError, match="the cache must serve"):
            DecodeLoop(args.pop("batch"), args.pop("vocab"), args.pop("dtype"), **args)


def _tool(name):
    path = os.path.join(LLVM, name)
    if not os.path.exists(path):
        pytest.skip(f"{name} not available")
    return path


def test_device_code_of_every_source(tmp_path):
    """Each source's code object: the library holds one bundle after the other."""
    fat = str(tmp_path / "fat.bin")
    subprocess.run([_tool("llvm-objcopy"), "--dump-section", f".hip_fatbin={fat}", binding.LIB_PATH, str(tmp_path / "x")],
                   check=True, capture_output=True)
    data = open(fat, "rb").read()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    kernels = []
    for n, at in enumerate(starts):
        part, co = str(tmp_path / f"{n}.bin"), str(tmp_path / f"{n}.o")
        with open(part, "wb") as f:
            f.write(data[at:starts[n + 1] if n + 1 < len(starts) else len(data)])
        subprocess.run([_tool("clang-offload-bundler"), "-type=o", "-targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                        f"-input={part}", f"-output={co}", "-unbundle"], check=True, capture_output=True)
        dis = subprocess.run([_tool("llvm-objdump"), "-d", co], check=True, capture_output=True, text=True).stdout
        assert "s_endpgm" in dis and not re.search(r"\bv_pk_(?:add|mul|fma)_f32\b", dis)
        notes = subprocess.run([_tool("llvm-readelf"), "--notes", co], check=True, capture_output=True, text=True).stdout
        names = re.findall(r"\.name:\s+(_Z\S+)", notes)
        scratch = [int(x) for x in re.findall(r"\.private_segment_fixed_size:\s+(\d+)", notes)]
        assert len(names) == len(scratch)
        assert not [x for x in zip(names, scratch) if x[1]]
        kernels += names
    for want in ("verify_kernel", "cache_plan_kernel", "cache_append_kernel", "attend_kernel"):
        assert any(want in k for k in kernels), want


def test_outputs_that_overlap_themselves_are_refused(lib):
    """Rows of the output that lie on one another (an expanded view) would be written by several workgroups at once;
    dimensions of one element may have any stride, and q may be expanded (it is only read)."""
    for i in range(3):
        strides = [1536, 512, 128]
        strides[i] = 0
        assert _attend(lib, out_stride=tuple(strides)) == PARAM, i
        # (up to here; no call may reach the GPU)
        assert _attend(lib, q_stride=tuple(strides), workspace_bytes=0) == WORKSPACE, i
    assert _attend(lib, batch=1, out_stride=(0, 512, 128), workspace_bytes=0) == WORKSPACE
    assert _attend(lib, max_new=1, out_stride=(512, 0, 128), workspace_bytes=0) == WORKSPACE
    assert _attend(lib, q_heads=1, kv_heads=1, out_stride=(1536, 512, 0), workspace_bytes=0) == WORKSPACE
