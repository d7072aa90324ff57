"""CPU-only: what bs_kvq_* and bs_token_logprobs refuse on the host, before anything is launched.  The pointers are made up; a call that
passes every check ends in BS_EHIP here, where no GPU is.  And what the compiled kernels hold in registers and wait for."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2605_08862_amd import binding as B
from paper_2605_08862_amd import build as BLD

P = 1 << 20          # an aligned address that nothing is read from


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("made-up device pointers")
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_08862_amd import build
        build.build()
    return B.lib()


def _desc(**over):
    d = dict(n_pages=8, n_slots=2, max_pages_per_seq=4, n_kv_heads=2, head_dim=128, k_pages=P, v_pages=P, k_scale=P, v_scale=P, block_table=P)
    d.update(over)
    return B.bs_kvq_desc(*[d[n] for n, _ in B.bs_kvq_desc._fields_])


BAD_DESC = [(dict(k_pages=0), B.BS_EINVAL), (dict(v_scale=0), B.BS_EINVAL), (dict(block_table=0), B.BS_EINVAL), (dict(k_pages=P + 8), B.BS_EINVAL),
            (dict(k_scale=P + 2), B.BS_EINVAL), (dict(head_dim=96), B.BS_ESHAPE), (dict(n_kv_heads=0), B.BS_ESHAPE), (dict(n_kv_heads=257), B.BS_ESHAPE),
            (dict(n_pages=0), B.BS_ESHAPE), (dict(n_slots=0), B.BS_ESHAPE), (dict(max_pages_per_seq=0), B.BS_ESHAPE)]


@pytest.mark.parametrize("name", ["bs_kvq_write", "bs_kvq_read"])
def test_copies(lib, name):
    def call(desc=None, n=2, slot=P, pos=P, rows=P, n_max=5, k=P, v=P, stride=256):
        d = C.byref(desc if desc is not None else _desc())
        return getattr(lib, name)(d, n, slot, pos, rows, n_max, k, v, stride, None, None)
    assert call() == B.BS_EHIP
    for over, want in BAD_DESC:
        assert call(desc=_desc(**over)) == want, over
    assert getattr(lib, name)(None, 2, P, P, P, 5, P, P, 256, None, None) == B.BS_EINVAL
    for over, want in [(dict(slot=None), B.BS_EINVAL), (dict(pos=None), B.BS_EINVAL), (dict(rows=None), B.BS_EINVAL), (dict(k=None), B.BS_EINVAL),
                       (dict(v=None), B.BS_EINVAL), (dict(k=P + 1), B.BS_EINVAL), (dict(n=0), B.BS_ESHAPE), (dict(n=4097), B.BS_ESHAPE), (dict(n_max=0), B.BS_ESHAPE),
                       (dict(n_max=257), B.BS_ESHAPE), (dict(stride=255), B.BS_ESHAPE), (dict(stride=-256), B.BS_ESHAPE)]:
        assert call(**over) == want, over
    assert call(n_max=256) == B.BS_EHIP                                        # all of a slot
    big = _desc(max_pages_per_seq=1 << 16)
    assert call(desc=big, n=4096, n_max=1 << 20) == B.BS_ESHAPE                # more workgroups than a launch has


def test_attention(lib):
    need = B.bs_kvq_workspace_bytes(6, 2, 128, 9)
    assert need > 0

    def call(desc=None, n=2, slot=P, ctx=P, rows=P, q_max=9, heads=6, q=P, stride=768, out=P, ws=P, nbytes=need):
        return lib.bs_kvq_attention(C.byref(desc if desc is not None else _desc()), n, slot, ctx, rows, q_max, heads, q, stride, out, None, ws, nbytes, None)
    assert call() == B.BS_EHIP
    for over, want in BAD_DESC:
        assert call(desc=_desc(**over)) == want, over
    for over, want in [(dict(slot=None), B.BS_EINVAL), (dict(ctx=None), B.BS_EINVAL), (dict(rows=None), B.BS_EINVAL), (dict(q=None), B.BS_EINVAL),
                       (dict(out=None), B.BS_EINVAL), (dict(ws=None), B.BS_EINVAL), (dict(q=P + 8), B.BS_EINVAL), (dict(out=P + 2), B.BS_EINVAL),
                       (dict(ws=P + 64), B.BS_EINVAL), (dict(stride=772), B.BS_EINVAL), (dict(stride=760), B.BS_ESHAPE), (dict(n=0), B.BS_ESHAPE),
                       (dict(n=4097), B.BS_ESHAPE), (dict(q_max=0), B.BS_ESHAPE), (dict(q_max=257), B.BS_ESHAPE), (dict(heads=5), B.BS_ESHAPE), (dict(heads=0), B.BS_ESHAPE),
                       (dict(nbytes=need - 1), B.BS_ECAPACITY)]:
        assert call(**over) == want, over
    for bad in [(5, 2, 128, 1), (0, 2, 128, 1), (6, 0, 128, 1), (6, 2, 96, 1), (6, 2, 128, 0), (129, 1, 64, 1), (512, 257, 64, 1)]:
        assert B.bs_kvq_workspace_bytes(*bad) == 0, bad
    assert B.bs_kvq_workspace_bytes(128, 1, 64, 1) > 0


def test_logprobs(lib):
    need = B.bs_token_logprobs_workspace_bytes(3, 4, 1000, 5)
    assert need > 0

    def call(n=3, vocab=1000, z=P, dtype=B.BS_F32, dl=None, k=4, tok=P, nt=None, t=1.0, top=5, lp=P, h=None, tt=P, tl=P, ws=P, nbytes=need):
        return lib.bs_token_logprobs(n, vocab, z, dtype, dl, k, tok, nt, t, top, lp, h, tt, tl, None, ws, nbytes, None)
    assert call() == B.BS_EHIP
    assert call(top=0, tt=None, tl=None) == B.BS_EHIP
    for over, want in [(dict(z=None), B.BS_EINVAL), (dict(tok=None), B.BS_EINVAL), (dict(lp=None), B.BS_EINVAL), (dict(ws=None), B.BS_EINVAL), (dict(tt=None), B.BS_EINVAL),
                       (dict(tl=None), B.BS_EINVAL), (dict(dtype=2), B.BS_EINVAL), (dict(dtype=-1), B.BS_EINVAL), (dict(t=0.0), B.BS_EINVAL), (dict(t=-1.0), B.BS_EINVAL),
                       (dict(t=float("nan")), B.BS_EINVAL), (dict(t=float("inf")), B.BS_EINVAL), (dict(t=1e-39), B.BS_EINVAL), (dict(z=P + 2), B.BS_EINVAL),
                       (dict(ws=P + 128), B.BS_EINVAL), (dict(vocab=1), B.BS_ESHAPE), (dict(vocab=(1 << 24) + 1), B.BS_ESHAPE), (dict(n=0), B.BS_ESHAPE),
                       (dict(n=4097), B.BS_ESHAPE), (dict(k=-1), B.BS_ESHAPE), (dict(k=4096), B.BS_ESHAPE), (dict(n=4096, k=300), B.BS_ESHAPE), (dict(top=33), B.BS_ESHAPE),
                       (dict(top=-1), B.BS_ESHAPE), (dict(vocab=4), B.BS_ESHAPE), (dict(nbytes=need - 1), B.BS_ECAPACITY)]:
        assert call(**over) == want, over
    assert call(z=P + 2, dtype=B.BS_BF16) == B.BS_EHIP
    for bad in [(0, 4, 1000, 5), (3, -1, 1000, 5), (3, 4, 1, 0), (3, 4, 1000, 33), (3, 4, 3, 4), (4096, 300, 1000, 5)]:
        assert B.bs_token_logprobs_workspace_bytes(*bad) == 0, bad


def test_bind_without_a_context(lib):
    assert lib.bs_kvq_bind_bytes(None) == 0 and lib.bs_kvq_bind(None, None, None, 0) == B.BS_EINVAL


def test_temperatures_whose_reciprocal_overflows(lib):
    need = B.bs_token_logprobs_workspace_bytes(1, 0, 100, 0)
    call = lambda t: lib.bs_token_logprobs(1, 100, P, B.BS_F32, None, 0, P, None, t, 0, P, None, None, None, None, P, need, None)
    assert all(call(t) == B.BS_EINVAL for t in (0.0, -1.0, 9e-39, 1e-45, float("inf"), float("nan")))
    assert call(1e-38) == call(3e38) == B.BS_EHIP


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    out = {}
    for name in ("kvq_attention", "logprob", "kvq"):
        path = tmp_path_factory.mktemp("asm") / (name + ".s")
        r = subprocess.run([hipcc, *BLD.FLAGS, "--offload-device-only", "-S", os.path.join(BLD.CSRC, name + ".hip"), "-o", str(path)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        out[name] = path.read_text()
    return out


def test_no_kernel_spills(assembly):
    """The accumulators, tiles and rows that the kernels keep in registers stay there."""
    spills = {n: int(s) for text in assembly.values() for n, s in re.findall(r"\.symbol:\s+(\S+)\.kd.*?\.vgpr_spill_count:\s+(\d+)", text, re.S)}
    assert len(spills) >= 18 and not any(spills.values()), spills


def test_requests_of_the_shared_tiles_are_counted_right(assembly):
    """The attention kernel for many rows waits for all but the N newest of its requests to memory, N a multiple of those of a tile: its loops hold these requests,
    and nothing else that counts."""
    loops = []
    for name, body in re.findall(r"^(\S*kvq_wide_kernelILi\d+\S*):[^\n]*\n(.*?)s_endpgm", assembly["kvq_attention"], re.S | re.M):
        D = int(re.search(r"ILi(\d+)", name)[1])
        for wait in re.finditer(r"s_waitcnt vmcnt\(([1-9]\d*)\) lgkmcnt\(0\)\n\ts_barrier", body):
            inside = []                                                       # backward branches over the wait: the innermost is its loop's
            for b in re.finditer(r"s_c?branch\S* (\.LBB\d+_\d+)", body[wait.start():]):
                end, start = wait.start() + b.end(), body.index("\n" + b[1] + ":")
                if start < wait.start():
                    inside.append((end - start, start, end))
            _, start, end = min(inside)
            ops = re.findall(r"^\t((?:global|buffer|flat|scratch)_\S+)", body[start:end], re.M)
            loops.append((D, int(wait[1]), sorted(ops)))
    expected = {(128, 5): 4, (128, 12): 2, (64, 3): 2, (64, 8): 1}         # (head size, N): sixteen-byte requests of a tile; and one for the scales
    assert len(loops) == 8
    for D, n, ops in loops:
        assert ops == ["global_load_lds_dword"] + ["global_load_lds_dwordx4"] * expected[D, n], (D, n, ops)


def test_a_cache_of_other_tensors_is_not_described():
    kv = dict(n_pages=5, n_slots=2, max_pages_per_seq=3, n_kv_heads=2, head_dim=64, k_pages=torch.zeros(5, 2 * 64 * 64, dtype=torch.uint8), v_pages=torch.zeros(5 * 2 * 64 * 64, dtype=torch.uint8),
              k_scale=torch.zeros(5, 2), v_scale=torch.zeros(5, 2), block_table=torch.zeros(2, 3, dtype=torch.int32))
    d = B.make_kvq_desc(kv)
    assert d.k_pages == kv["k_pages"].data_ptr() and d.block_table == kv["block_table"].data_ptr() and d.n_pages == 5
    for name in ("k_pages", "v_pages", "k_scale", "v_scale", "block_table"):
        t = kv[name]
        for bad in (t.flatten()[:-1], t.to(torch.int64), t.to(torch.bfloat16), torch.cat([t, t])[::2], t.to("meta")):
            with pytest.raises(B.BsError) as e:
                B.make_kvq_desc(dict(kv, **{name: bad}))
            assert e.value.status == B.BS_EINVAL, name
