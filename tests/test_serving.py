"""CPU tests of cr_append_kv and cr_attend: argument checks (every call here
returns before anything is enqueued), the workspace, and the host code under
the address and undefined-behaviour sanitizers."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2609_35139_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = float


def _batch(L=2, H=2, d=64, dtype=B.CR_DTYPE_BF16, n_seqs=3, bs=16, max_blocks=8, n_blocks=30,
           offsets=(0, 2, 2, 9), lens=0x7000, table=0x8000):
    lay, sB = B.paged_layout(L, H, d, n_blocks, bs, dtype)
    q, keep = B.sequences_struct(n_seqs, lens, table, max_blocks, bs, n_blocks, sB, offsets)
    q.keep = keep
    return lay, q


def _rows(heads=4, d=64, data=0x100000, token=None, head=None):
    return B.cr_rows(data, heads * d if token is None else token, d if head is None else head)


def _append(lay, q, kv=0x10000, layer=1, k=None, v=None, qr=None, qo=None, heads=4, rope=None,
            positions=None):
    with pytest.raises(B.CrError) as e:
        B.cr_append_kv(kv, lay, layer, q, k or _rows(2, lay.head_dim, 0x200000),
                       v or _rows(2, lay.head_dim, 0x300000), qr, qo, heads, rope, positions)
    return e.value.name


def _attend(lay, q, kv=0x10000, layer=1, qr=None, out=None, heads=4, ws=0x400000, ws_bytes=1 << 40, **o):
    opt = B.cr_attend_options()
    for k, x in o.items():
        setattr(opt, k, x)
    with pytest.raises(B.CrError) as e:
        B.cr_attend(kv, lay, layer, q, qr or _rows(heads, lay.head_dim), out or _rows(heads, lay.head_dim, 0x500000),
                    heads, opt, ws, ws_bytes)
    return e.value.name


def test_struct_sizes_match_c():
    assert ctypes.sizeof(B.cr_sequences) == 56
    assert ctypes.sizeof(B.cr_rows) == 24
    assert ctypes.sizeof(B.cr_attend_options) == 48


@pytest.mark.parametrize("call", [_append, _attend])
@pytest.mark.parametrize("change,name", [
    (dict(n_seqs=0, offsets=(0,)), "CR_ERR_OFFSETS"),
    (dict(offsets=(1, 2, 2, 9)), "CR_ERR_OFFSETS"),
    (dict(offsets=(0, 2, 1, 9)), "CR_ERR_OFFSETS"),
    (dict(lens=0), "CR_ERR_NULL"),
    (dict(table=0), "CR_ERR_NULL"),
    (dict(dtype=2), "CR_ERR_DTYPE"),
    (dict(d=48), "CR_ERR_DIMS"),
    (dict(d=288), "CR_ERR_DIMS"),
    (dict(bs=3), "CR_ERR_LAYOUT"),
    (dict(bs=2048), "CR_ERR_LAYOUT"),
    (dict(bs=1024, max_blocks=1 << 21), "CR_ERR_LAYOUT"),     # slots past 2^31 - 256
    (dict(max_blocks=0), "CR_ERR_LAYOUT"),
    (dict(n_blocks=0), "CR_ERR_LAYOUT"),
])
def test_bad_batches(call, change, name):
    assert call(*_batch(**change)) == name


@pytest.mark.parametrize("call", [_append, _attend])
def test_bad_caches(call):
    lay, q = _batch()
    assert call(lay, q, kv=0) == "CR_ERR_NULL"
    assert call(lay, q, kv=0x10008) == "CR_ERR_LAYOUT"
    assert call(lay, q, layer=2) == "CR_ERR_DIMS"
    assert call(lay, q, layer=-1) == "CR_ERR_DIMS"
    q.stride_block += 4
    assert call(lay, q) == "CR_ERR_LAYOUT"
    lay, q = _batch()
    q.stride_block = lay.stride_token                          # blocks overlap
    assert call(lay, q) == "CR_ERR_LAYOUT"
    lay, q = _batch()
    lay.stride_token = -lay.stride_token
    assert call(lay, q) == "CR_ERR_LAYOUT"


@pytest.mark.parametrize("bad", [_rows(2, 64, 0x200008), _rows(2, 64, token=132), _rows(2, 64, head=68),
                                 _rows(2, 64, token=-128), _rows(2, 64, token=1 << 61),
                                 _rows(2, 64, token=(1 << 62) - 8)])
def test_bad_rows(bad):
    lay, q = _batch()
    ok = _rows(2, 64, 0x600000)
    assert _append(lay, q, k=bad) == "CR_ERR_LAYOUT"
    assert _append(lay, q, v=bad) == "CR_ERR_LAYOUT"
    assert _append(lay, q, qr=bad, qo=ok, heads=2) == "CR_ERR_LAYOUT"
    assert _append(lay, q, qr=ok, qo=bad, heads=2) == "CR_ERR_LAYOUT"
    assert _attend(lay, q, qr=bad, heads=2) == "CR_ERR_LAYOUT"
    assert _attend(lay, q, out=bad, heads=2) == "CR_ERR_LAYOUT"


def test_bad_operands():
    lay, q = _batch()
    a, b = _rows(4, 64, 0x600000), _rows(4, 64, 0x700000)
    assert _append(lay, q, qr=a) == "CR_ERR_NULL"              # q without q_out
    assert _append(lay, q, qo=a) == "CR_ERR_NULL"
    assert _append(lay, q, k=B.cr_rows(0, 128, 64)) == "CR_ERR_NULL"
    assert _append(lay, q, qr=a, qo=b, heads=0) == "CR_ERR_DIMS"
    overlap = _rows(4, 64, 0x700000, token=0)                  # written rows on top of each other
    assert _append(lay, q, qr=a, qo=overlap) == "CR_ERR_LAYOUT"
    assert _attend(lay, q, out=overlap) == "CR_ERR_LAYOUT"
    shifted = _rows(4, 64, 0x600000, token=512)                # in place with other strides
    assert _append(lay, q, qr=a, qo=shifted) == "CR_ERR_LAYOUT"
    assert _attend(lay, q, qr=a, out=a) == "CR_ERR_LAYOUT"
    for rope in (dict(theta=0.0), dict(scale=0.0), dict(scale=F("inf")), dict(inv_freq=[F("nan")] * 32)):
        r, keep = B.rope_struct(**rope)
        assert _append(lay, q, rope=r) == "CR_ERR_DIMS", rope
        del keep


@pytest.mark.parametrize("o", [dict(scale=-1.0), dict(scale=F("nan")), dict(scale=F("inf")),
                               dict(softcap=-1.0), dict(softcap=F("nan")), dict(softcap=F("inf")),
                               dict(shared_len=-1), dict(shared_len=129)])
def test_bad_attend_options(o):
    assert _attend(*_batch(), **o) == "CR_ERR_DIMS"


def test_bad_heads_slopes_and_workspace():
    lay, q = _batch()
    for heads in (0, 3, -2, 258):
        assert _attend(lay, q, heads=heads) == "CR_ERR_DIMS"
    s = (ctypes.c_float * 4)(0.1, F("nan"), 0, 0)
    assert _attend(lay, q, slopes=ctypes.cast(s, ctypes.POINTER(ctypes.c_float))) == "CR_ERR_DIMS"
    lay, q = _batch(bs=1024)
    need = B.cr_attend_workspace_bytes(lay, q, 4)
    assert need > 0
    assert _attend(lay, q, ws_bytes=need - 1) == "CR_ERR_WORKSPACE"
    assert _attend(lay, q, ws=0x400080) == "CR_ERR_WORKSPACE"
    assert _attend(lay, q, ws=0) == "CR_ERR_NULL"
    assert B.cr_attend_workspace_bytes(lay, q, 4, 100) == need     # a pass of its own would not pay
    with pytest.raises(B.CrError):
        B.cr_attend_workspace_bytes(lay, q, 4, 1 << 20)


def test_a_batch_without_tokens_is_a_no_op():
    lay, q = _batch(offsets=(0, 0, 0, 0))
    empty = B.cr_rows(None, 0, 0)
    B.cr_append_kv(0x10000, lay, 0, q, empty, empty, empty, empty, 4, None, None)
    assert B.cr_attend_workspace_bytes(lay, q, 4) == 0
    B.cr_attend(0x10000, lay, 0, q, empty, B.cr_rows(0x10000, 0, 0), 4, None, None, 0)


def test_offsets_are_the_batch_s_own():
    off = np.array([0, 2, 5], dtype=np.int32)
    q, keep = B.sequences_struct(2, 0x1000, 0x2000, 4, 16, 8, 16 * 128, off)
    off[:] = 99
    assert [q.query_offsets[i] for i in range(3)] == [0, 2, 5] == keep.tolist()


def test_workspace_does_not_grow_with_the_table():
    """The split is bounded by the chip, not by the longest context there can be."""
    sizes = []
    for blocks in (1 << 10, 1 << 16):
        lay, q = _batch(max_blocks=blocks, offsets=None)
        sizes.append(B.cr_attend_workspace_bytes(lay, q, 4))
    assert sizes[0] == sizes[1] < 1 << 28
    assert sizes[1] < B.cr_attend_workspace_bytes(lay, q, 4, 1 << 19) < 1 << 28


# Host-only sanitizer build of the entry points, linked against launchers that
# always fail, driven by a deterministic fuzzer (tests/sanitize/serve_fuzz.cpp).
def test_host_code_is_clean_under_address_and_ub_sanitizers(tmp_path):
    try:
        import torch
        if torch.cuda.is_available():
            pytest.skip("host-only check; the fuzzer refuses to run where a GPU is visible")
    except ImportError:
        pass
    from test_abi import SAN_COMPILE, SAN_LINK
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    compiler = os.path.join(rocm, "bin", "hipcc")
    linker = os.path.join(rocm, "llvm", "bin", "clang++")
    if not (os.path.exists(compiler) and os.path.exists(linker)):
        pytest.skip("ROCm toolchain not found")
    csrc, san = os.path.join(ROOT, "paper_2609_35139_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize")
    objs = []
    for src in (os.path.join(csrc, "serve.hip"), os.path.join(san, "serve_stubs.hip"),
                os.path.join(san, "serve_fuzz.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run([compiler, "--offload-arch=gfx950", *SAN_COMPILE, "-I",
                            os.path.join(ROOT, "include"), "-c", src, "-o", obj],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        objs.append(obj)
    exe = str(tmp_path / "serve_fuzz")
    r = subprocess.run([linker, *SAN_LINK, *objs, "-L", os.path.join(rocm, "lib"), "-lamdhip64",
                        "-Wl,-rpath," + os.path.join(rocm, "lib"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe, "20000"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
    counts = dict(kv.split(":") for kv in r.stdout.split("counts:")[1].split())
    assert int(counts["-7"]) > 1000          # reached the device check: fully validated
    for code in ("0", "-1", "-2", "-3", "-4", "-5", "-6"):
        assert int(counts[code]) > 0, code   # each rejection path, and sizes, exercised
