"""CPU tests of cr_weigh_keys, cr_choose_slots, cr_compact_kv and cr_sample:
argument checks (every call here returns before anything is enqueued), the
workspace, and the host code under the address and undefined-behaviour
sanitizers."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_35139_amd import binding as B
from test_serving import _batch, _rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = float


def _weights(L=2, S=3, H=2, slots=128, data=0x900000, layer=None, seq=None, head=None):
    return B.cr_key_weights(data, S * H * slots if layer is None else layer,
                            H * slots if seq is None else seq, slots if head is None else head)


def _weigh(lay, q, kv=0x10000, layer=1, qr=None, heads=4, w=None, options=True, lse=0x800000,
           ws=0x400000, ws_bytes=1 << 40, **o):
    opt = B.cr_attend_options()
    opt.lse = lse
    for k, x in o.items():
        setattr(opt, k, x)
    with pytest.raises(B.CrError) as e:
        B.cr_weigh_keys(kv, lay, layer, q, qr or _rows(heads, lay.head_dim), heads,
                        opt if options else None,
                        w or _weights(lay.n_layers, q.n_seqs, lay.n_kv_heads,
                                      max(q.max_blocks * q.block_size, 1)), ws, ws_bytes)
    return e.value.name


def _choose(lay, q, w=None, budget=8, first=1, recent=2, kept=0xa00000, lens=0xb00000, budgets=None):
    with pytest.raises(B.CrError) as e:
        B.cr_choose_slots(lay, q, w or _weights(lay.n_layers, q.n_seqs, lay.n_kv_heads,
                                                max(q.max_blocks * q.block_size, 1)),
                          B.cr_choice(budget, first, recent, budgets), kept, lens)
    return e.value.name


def _compact(lay, q, kv=0x10000, kept=0xa00000, budget=8, lens=0xb00000, out=None, blocks=0, w=None):
    with pytest.raises(B.CrError) as e:
        B.cr_compact_kv(kv, lay, q, kept, budget, lens, out, blocks, w)
    return e.value.name


def _sample(data=0x100000, dtype=B.CR_DTYPE_F32, rows=3, vocab=1000, stride=1000, options=None,
            u=0x200000, tokens=0x300000, log_probs=None):
    with pytest.raises(B.CrError) as e:
        B.cr_sample(B.cr_logits(data, dtype, rows, vocab, stride), options, u, tokens, log_probs)
    return e.value.name


def test_struct_sizes_match_c():
    assert ctypes.sizeof(B.cr_key_weights) == 32
    assert ctypes.sizeof(B.cr_choice) == 24
    assert ctypes.sizeof(B.cr_logits) == 32
    assert ctypes.sizeof(B.cr_sampling) == 48


@pytest.mark.parametrize("change,name", [
    (dict(n_seqs=0, offsets=(0,)), "CR_ERR_OFFSETS"),
    (dict(offsets=(1, 2, 2, 9)), "CR_ERR_OFFSETS"),
    (dict(offsets=(0, 2, 1, 9)), "CR_ERR_OFFSETS"),
    (dict(lens=0), "CR_ERR_NULL"),
    (dict(table=0), "CR_ERR_NULL"),
    (dict(dtype=2), "CR_ERR_DTYPE"),
    (dict(d=48), "CR_ERR_DIMS"),
    (dict(bs=3), "CR_ERR_LAYOUT"),
    (dict(bs=1024, max_blocks=1 << 21), "CR_ERR_LAYOUT"),
    (dict(max_blocks=0), "CR_ERR_LAYOUT"),
    (dict(n_blocks=0), "CR_ERR_LAYOUT"),
])
def test_bad_batches_of_weigh(change, name):
    assert _weigh(*_batch(**change)) == name


@pytest.mark.parametrize("call", [_choose, _compact])
@pytest.mark.parametrize("change,name", [
    (dict(n_seqs=0, offsets=None), "CR_ERR_OFFSETS"),
    (dict(L=0), "CR_ERR_DIMS"),
    (dict(H=0), "CR_ERR_DIMS"),
    (dict(lens=0), "CR_ERR_NULL"),
    (dict(bs=3), "CR_ERR_LAYOUT"),
    (dict(max_blocks=0), "CR_ERR_LAYOUT"),
    (dict(bs=1024, max_blocks=(1 << 20) + 1), "CR_ERR_DIMS"),         # more than 2^30 slots
    (dict(L=1 << 12, n_seqs=1 << 11, offsets=None), "CR_ERR_DIMS"),   # 2^32 threads
])
def test_bad_sequences(call, change, name):
    assert call(*_batch(**change)) == name


def test_bad_weights():
    lay, q = _batch()
    for w, name in ((_weights(data=0), "CR_ERR_NULL"), (_weights(data=0x900002), "CR_ERR_LAYOUT"),
                    (_weights(head=127), "CR_ERR_LAYOUT"), (_weights(seq=-256), "CR_ERR_LAYOUT"),
                    (_weights(layer=0), "CR_ERR_LAYOUT"), (_weights(layer=1 << 62), "CR_ERR_LAYOUT")):
        assert _weigh(lay, q, w=w) == name
        assert _choose(lay, q, w=w) == name
        assert _compact(lay, q, w=w) == name


def test_bad_weigh_calls():
    lay, q = _batch()
    assert _weigh(lay, q, kv=0) == "CR_ERR_NULL"
    assert _weigh(lay, q, options=False) == "CR_ERR_NULL"
    assert _weigh(lay, q, lse=None) == "CR_ERR_NULL"
    assert _weigh(lay, q, kv=0x10008) == "CR_ERR_LAYOUT"
    assert _weigh(lay, q, layer=2) == "CR_ERR_DIMS"
    assert _weigh(lay, q, qr=_rows(4, 64, 0x200008)) == "CR_ERR_LAYOUT"
    assert _weigh(lay, q, qr=B.cr_rows(0, 256, 64)) == "CR_ERR_NULL"
    for heads in (0, 3, 258):
        assert _weigh(lay, q, heads=heads) == "CR_ERR_DIMS"
    for o in (dict(scale=-1.0), dict(scale=F("inf")), dict(softcap=F("nan")), dict(shared_len=-1)):
        assert _weigh(lay, q, **o) == "CR_ERR_DIMS"
    # a prompt: what its rows bring lies in the workspace
    lay, q = _batch(offsets=(0, 2, 2, 900))
    need = B.cr_weigh_workspace_bytes(lay, q, 4)
    assert need > 900 * 4 * 32
    assert _weigh(lay, q, ws_bytes=need - 1) == "CR_ERR_WORKSPACE"
    assert _weigh(lay, q, ws=0x400080) == "CR_ERR_WORKSPACE"
    assert _weigh(lay, q, ws=0) == "CR_ERR_NULL"


def test_single_tokens_take_no_workspace():
    lay, q = _batch(offsets=None)
    assert B.cr_weigh_workspace_bytes(lay, q, 4) == 0
    assert _weigh(lay, q, ws=0, ws_bytes=0) == "CR_ERR_DEVICE" if not torch.cuda.is_available() else True


def test_a_batch_without_tokens_is_a_no_op():
    lay, q = _batch(offsets=(0, 0, 0, 0))
    opt = B.cr_attend_options()
    assert B.cr_weigh_workspace_bytes(lay, q, 4) == 0
    B.cr_weigh_keys(0x10000, lay, 0, q, B.cr_rows(None, 0, 0), 4, opt, _weights(), None, 0)
    B.cr_sample(B.cr_logits(None, B.CR_DTYPE_BF16, 0, 1000, 1000), None, None, None, None)


def test_bad_choices():
    lay, q = _batch()
    assert _choose(lay, q, budget=0) == "CR_ERR_DIMS"
    assert _choose(lay, q, first=-1) == "CR_ERR_DIMS"
    assert _choose(lay, q, recent=-1) == "CR_ERR_DIMS"
    assert _choose(lay, q, kept=0) == "CR_ERR_NULL"
    assert _choose(lay, q, lens=0) == "CR_ERR_NULL"


def test_lists_past_what_their_indexes_hold():
    lay, q = _batch()
    assert _choose(lay, q, budget=(1 << 30) + 1) == "CR_ERR_DIMS"
    assert _compact(lay, q, budget=(1 << 31) - 1) == "CR_ERR_DIMS"


def test_lengths_after_in_the_lengths_before():
    """Sequences' workgroups would read lengths that another one has written; a compaction
    would take the new lengths for the old ones."""
    lay, q = _batch()
    for at in (0, 4, -4):
        assert _choose(lay, q, lens=q.kv_lens + at) == "CR_ERR_LAYOUT"
        assert _compact(lay, q, lens=q.kv_lens + at) == "CR_ERR_LAYOUT"
        assert _choose(lay, q, lens=0xd00000 + at, budgets=0xd00000) == "CR_ERR_LAYOUT"
    if torch.cuda.is_available():
        return
    for at in (4 * q.n_seqs, -4 * q.n_seqs):                   # next to each other
        assert _choose(lay, q, lens=q.kv_lens + at) == "CR_ERR_DEVICE"
        assert _compact(lay, q, lens=q.kv_lens + at) == "CR_ERR_DEVICE"


def test_settings_that_32_bits_do_not_hold():
    """A limit of 2^32 + 1 tokens is not one of one token."""
    from paper_2609_35139_amd.serving import _int32
    assert [_int32(v) for v in (0, -3, 7, (1 << 32) + 1, -(1 << 40), (1 << 31) - 1)] == \
        [0, -3, 7, (1 << 31) - 1, -(1 << 31), (1 << 31) - 1]


def test_bad_compactions():
    lay, q = _batch()
    assert _compact(lay, q, kv=0) == "CR_ERR_NULL"
    assert _compact(lay, q, kept=0) == "CR_ERR_NULL"
    assert _compact(lay, q, lens=0) == "CR_ERR_NULL"
    assert _compact(lay, q, budget=0) == "CR_ERR_DIMS"
    assert _compact(lay, q, kv=0x10008) == "CR_ERR_LAYOUT"
    assert _compact(lay, q, out=0xc00000, blocks=0) == "CR_ERR_LAYOUT"
    assert _compact(lay, q, out=0xc00000, blocks=1 << 28) == "CR_ERR_LAYOUT"
    lay.dtype = 5
    assert _compact(lay, q) == "CR_ERR_DTYPE"
    lay, q = _batch()
    q.stride_block = lay.stride_token                          # blocks overlap
    assert _compact(lay, q) == "CR_ERR_LAYOUT"


@pytest.mark.parametrize("change,name", [
    (dict(dtype=2), "CR_ERR_DTYPE"), (dict(rows=-1), "CR_ERR_DIMS"), (dict(rows=1 << 22), "CR_ERR_DIMS"),
    (dict(vocab=0), "CR_ERR_DIMS"), (dict(vocab=(1 << 19) + 1), "CR_ERR_DIMS"),
    (dict(stride=-8), "CR_ERR_LAYOUT"), (dict(stride=1 << 60), "CR_ERR_LAYOUT"),
    (dict(data=0x100002), "CR_ERR_LAYOUT"), (dict(data=0x100001, dtype=B.CR_DTYPE_BF16), "CR_ERR_LAYOUT"),
    (dict(data=None), "CR_ERR_NULL"), (dict(u=None), "CR_ERR_NULL"), (dict(tokens=None), "CR_ERR_NULL"),
])
def test_bad_logits(change, name):
    assert _sample(**change) == name


def test_sample_refuses_host_tensors():
    from paper_2609_35139_amd.serving import sample
    with pytest.raises(TypeError):
        sample(torch.zeros(2, 10), torch.zeros(2))


# Host-only sanitizer build of the entry points, linked against launchers that
# always fail, driven by a deterministic fuzzer (tests/sanitize/answer_fuzz.cpp).
def test_host_code_is_clean_under_address_and_ub_sanitizers(tmp_path):
    if torch.cuda.is_available():
        pytest.skip("host-only check; the fuzzer refuses to run where a GPU is visible")
    from test_abi import SAN_COMPILE, SAN_LINK
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    compiler = os.path.join(rocm, "bin", "hipcc")
    linker = os.path.join(rocm, "llvm", "bin", "clang++")
    if not (os.path.exists(compiler) and os.path.exists(linker)):
        pytest.skip("ROCm toolchain not found")
    csrc, san = os.path.join(ROOT, "paper_2609_35139_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize")
    objs = []
    for src in (os.path.join(csrc, "answer.hip"), os.path.join(san, "answer_stubs.hip"),
                os.path.join(san, "answer_fuzz.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run([compiler, "--offload-arch=gfx950", *SAN_COMPILE, "-I",
                            os.path.join(ROOT, "include"), "-c", src, "-o", obj],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        objs.append(obj)
    exe = str(tmp_path / "answer_fuzz")
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
        assert int(counts[code]) > 0, code
