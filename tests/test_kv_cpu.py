"""The paged MXFP4 cache without a GPU: layout and cutting of work replayed on the host, and calls that are refused before a
device is touched."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_08713_amd", "csrc")
CHECK = os.path.join(ROOT, "tests", "kv_layout_check.cpp")
OK, EINVAL, ENULL, EALIGN, EUNSUPPORTED = 0, -1, -2, -3, -4
A = 0x10000  # a fake device address, aligned to everything


@pytest.fixture(scope="module")
def lib():
    from paper_2603_08713_amd import binding
    from paper_2603_08713_amd import build as mxbuild

    if not os.path.exists(mxbuild.LIB):
        mxbuild.build()
    return binding.load_library()


def _replay(tmp_path, include):
    exe = str(tmp_path / "check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", include, CHECK, "-o", exe], check=True, stderr=subprocess.PIPE, text=True)
    return subprocess.run([exe], stdout=subprocess.PIPE, text=True)


def test_layout_requests_and_pieces(tmp_path):
    out = _replay(tmp_path, CSRC)
    assert out.returncode == 0 and "hold" in out.stdout, out.stdout[-2000:]


@pytest.mark.parametrize("right, wrong", [
    ("unit * 16 + (place & 3) * 4", "unit * 16 + (place & 1) * 4"),                                    # two tokens on the same bytes
    ("kv_clamp(end, r.first, T) - r.first", "kv_clamp(end, r.first, T + 1) - r.first"),                # a row behind the tensor
    ("kv_min(pos0 + i, kKvMostKeys) - (window - 1)", "kv_min(pos0 + i, kKvMostKeys) - window"),        # a window of one key more
    ("(uint32_t)(at + item - 1) / (uint32_t)share", "(uint32_t)(at + item) / (uint32_t)share"),        # a part too many
    ("(total + ((int64_t)1 << workers_log2) - 1)", "(total)"),                                         # the last tiles are lost
    ("2 * worker + (at > begin)", "2 * worker"),                                                       # two results in one place
    ("if ((at + item) >> 32)", "if ((at + item) >> 40)"),                                              # positions cut off
])
def test_a_planted_mistake_is_found(tmp_path, right, wrong):
    text = open(os.path.join(CSRC, "mx_kv_layout.h")).read()
    assert text.count(right) == 1
    (tmp_path / "mx_kv_layout.h").write_text(text.replace(right, wrong))
    out = _replay(tmp_path, str(tmp_path))
    assert out.returncode != 0


def _changed(base, **changes):
    assert set(changes) <= set(base)
    return list(dict(base, **changes).values())


PLAN = dict(ctx=A, new=A + 64, S=4, page=64, table=A, max_pages=8, free=A, count=9, start=A + 4, T=10, offsets=A, lens=A + 128, slots=A,
            positions=A, next=A, stream=None)
CACHE = dict(kc=A, ks=A, km=A, vc=A, vs=A, vm=A, pages=5, page=64)
TURN = dict(q=A, ldq=1024, k=A, ldk=256, positions=A, table=A, most=100, qw=A, kw=A, eps=1e-6, style=0, T=3, Hq=8, Hkv=2, D=128, R=128, q_out=A,
            ldqo=1024, k_out=A, ldko=256, stream=None)
WRITE = dict(k=A, ldk=256, v=A, ldv=256, slots=A, rule=2, **CACHE, T=3, Hkv=2, D=128, stream=None)
BOTH = dict(q=A, ldq=1024, k=A, ldk=256, v=A, ldv=256, positions=A, table=A, most=100, qw=A, kw=A, eps=1e-6, style=0, slots=A, rule=2, **CACHE, T=3,
            Hq=8, Hkv=2, D=128, R=128, q_out=A, ldqo=1024, stream=None)
READ = dict(slots=A, **CACHE, T=3, Hkv=2, D=128, dtype=1, k_out=A, ldk=256, v_out=A, ldv=256, stream=None)
ATTEND = dict(q=A, ldq=1024, offsets=A, lens=A, table=A, max_pages=8, **CACHE, S=2, T=3, Hq=8, Hkv=2, D=128, scale=0.1, causal=1, window=0, out=A,
              ldo=1024, lse=None, work=A, bytes=1 << 40, stream=None)

BAD_CACHE = [(dict(kc=None), ENULL), (dict(vs=None), ENULL), (dict(km=None), EINVAL), (dict(vm=None), EINVAL), (dict(kc=A + 8), EALIGN), (dict(vs=A + 2), EALIGN),
             (dict(page=48), EUNSUPPORTED), (dict(page=8), EUNSUPPORTED), (dict(page=8192), EUNSUPPORTED), (dict(page=0), EINVAL), (dict(pages=-1), EINVAL),
             (dict(pages=1 << 50), EINVAL), (dict(pages=1 << 62), EINVAL), (dict(D=80), EUNSUPPORTED), (dict(D=160), EUNSUPPORTED), (dict(D=0), EUNSUPPORTED)]
BAD_TURN = [(dict(T=-1), EINVAL), (dict(T=1 << 31), EINVAL), (dict(Hq=-1), EINVAL), (dict(ldq=1016), EINVAL), (dict(ldk=248), EINVAL), (dict(ldqo=8), EINVAL),
            (dict(q=None), ENULL), (dict(k=None), ENULL), (dict(q_out=None), ENULL), (dict(positions=None), ENULL), (dict(table=None), EINVAL), (dict(R=0), EINVAL),
            (dict(R=144), EINVAL), (dict(R=24), EUNSUPPORTED), (dict(style=2), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
            (dict(q=A + 8), EALIGN), (dict(ldk=260), EALIGN), (dict(table=A + 8), EALIGN), (dict(kw=A + 2), EALIGN), (dict(most=-1), EINVAL), (dict(D=144), EUNSUPPORTED)]


@pytest.mark.parametrize("name, base, bad", [
    ("mx_kv_plan", PLAN, [(dict(S=-1), EINVAL), (dict(S=5000), EUNSUPPORTED), (dict(page=24), EUNSUPPORTED), (dict(page=-16), EINVAL), (dict(T=-1), EINVAL),
                          (dict(max_pages=1 << 40), EINVAL), (dict(max_pages=1 << 62), EINVAL), (dict(max_pages=-1), EINVAL), (dict(ctx=None), ENULL), (dict(slots=None), ENULL), (dict(free=None), ENULL),
                          (dict(start=None), ENULL), (dict(next=A + 4), EINVAL), (dict(lens=A), EINVAL), (dict(lens=A + 64), EINVAL), (dict(offsets=A + 4), EALIGN),
                          (dict(count=1 << 40), EINVAL), (dict(table=None), ENULL)]),
    ("mx_qk_norm_rope", TURN, BAD_TURN + [(dict(k_out=None), ENULL), (dict(ldko=128), EINVAL), (dict(k_out=A + 2), EALIGN)]),
    ("mx_kv_write", WRITE, BAD_CACHE + [(dict(k=None), ENULL), (dict(slots=None), ENULL), (dict(rule=3), EINVAL), (dict(T=-1), EINVAL), (dict(ldv=255), EINVAL),
                                        (dict(ldv=257), EALIGN), (dict(slots=A + 4), EALIGN), (dict(Hkv=0), EINVAL)]),
    ("mx_qk_norm_rope_kv_write", BOTH, BAD_CACHE + BAD_TURN + [(dict(v=None), ENULL), (dict(slots=None), ENULL), (dict(rule=-1), EINVAL), (dict(v=A + 4), EALIGN)]),
    ("mx_kv_read", READ, BAD_CACHE + [(dict(slots=None), ENULL), (dict(k_out=None, v_out=None), ENULL), (dict(dtype=2), EINVAL), (dict(ldk=128), EINVAL),
                                      (dict(k_out=A + 8), EALIGN)]),
    ("mx_attention_kv", ATTEND, BAD_CACHE + [(dict(q=None), ENULL), (dict(out=None), ENULL), (dict(lens=None), ENULL), (dict(table=None), ENULL), (dict(S=-1), EINVAL),
                                             (dict(T=-2), EINVAL), (dict(Hq=7), EINVAL), (dict(window=-1), EINVAL), (dict(causal=0, window=5), EINVAL), (dict(bytes=0), EINVAL),
                                             (dict(work=None), ENULL), (dict(work=A + 4), EALIGN), (dict(q=A + 2), EALIGN), (dict(ldo=1000), EINVAL), (dict(ldq=1028), EALIGN),
                                             (dict(max_pages=1 << 30), EINVAL), (dict(Hkv=0), EINVAL)]),
])
def test_refusals(lib, name, base, bad):
    call = getattr(lib, name)
    assert len(base) == len(call.argtypes)
    for changes, status in bad:
        assert call(*_changed(base, **changes)) == status, (name, changes)


B = 1 << 20  # bytes between arrays that lie apart
APART = dict(PLAN, ctx=A, new=A + B, table=A + 2 * B, free=A + 3 * B, start=A + 4 * B, offsets=A + 5 * B, lens=A + 6 * B, slots=A + 7 * B, positions=A + 8 * B,
             next=A + 9 * B)


@pytest.mark.parametrize("out, size", [("table", 128), ("offsets", 40), ("lens", 16), ("slots", 80), ("positions", 40), ("next", 4)])
@pytest.mark.parametrize("into, length", [("ctx", 16), ("new", 16), ("free", 36), ("start", 4)])
def test_a_plan_does_not_write_what_it_reads(lib, out, size, into, length):
    """Workgroups read the lengths and the free list while others write: an output on any byte of theirs is refused, one right beside them is not."""
    step = 8 if out in ("offsets", "slots") else 4
    at = APART[into]
    for address in range(at - size // step * step + step, at + length, step):
        assert lib.mx_kv_plan(*_changed(APART, **{out: address})) == EINVAL, address - at
    import torch

    if not torch.cuda.device_count():  # (the addresses are made up)
        for address in (at - size, at + -(-length // step) * step):
            assert lib.mx_kv_plan(*_changed(APART, **{out: address})) == EUNSUPPORTED, address - at


def test_empty_calls_do_nothing(lib):
    """No tokens, no requests or no pages: nothing is launched, so no device is needed."""
    assert lib.mx_qk_norm_rope(*_changed(TURN, T=0)) == OK
    assert lib.mx_qk_norm_rope(*_changed(TURN, Hq=0, Hkv=0)) == OK
    assert lib.mx_kv_write(*_changed(WRITE, T=0)) == OK
    assert lib.mx_kv_write(*_changed(WRITE, pages=0, kc=None, ks=None, km=None, vc=None, vs=None, vm=None)) == OK
    assert lib.mx_qk_norm_rope_kv_write(*_changed(BOTH, T=0)) == OK
    assert lib.mx_kv_read(*_changed(READ, T=0)) == OK
    assert lib.mx_attention_kv(*_changed(ATTEND, T=0)) == OK
    assert lib.mx_attention_kv(*_changed(ATTEND, S=0)) == OK


# (a wavefront has 8, 4 or 2 tokens of up to eight heads of queries, keys or values; a workgroup has four wavefronts)
@pytest.mark.parametrize("name, base, changes, most", [
    ("mx_qk_norm_rope", TURN, dict(Hq=1, Hkv=0, D=256), 2 * ((1 << 26) - 4)),
    ("mx_qk_norm_rope", TURN, dict(Hq=0, Hkv=9, ldk=1152, ldko=1152), 4 * ((1 << 25) - 2)),
    ("mx_kv_write", WRITE, dict(Hkv=1, D=256), 2 * ((1 << 25) - 2)),
    ("mx_qk_norm_rope_kv_write", BOTH, dict(Hq=1, Hkv=1, D=256), 2 * ((1 << 26) // 3 - 1)),
    ("mx_kv_read", READ, dict(Hkv=1, D=256), 2 * ((1 << 25) - 2)),
    ("mx_attention_kv", ATTEND, dict(Hq=1, Hkv=1, S=1 << 26), (1 << 26) - 4),
    ("mx_attention_kv", ATTEND, dict(Hq=1, Hkv=1, S=1), (1 << 30) - 1),
    ("mx_attention_kv", ATTEND, dict(Hq=8, Hkv=8, S=1), 256 * ((1 << 20) - 2)),
])
def test_the_largest_launches(lib, name, base, changes, most):
    """A launch holds fewer than 2^32 work-items, its last workgroup whole.  What would not fit is refused with the arguments, before anything runs."""
    torch = pytest.importorskip("torch")
    call = getattr(lib, name)
    for T in (most + 1, most + 4, most + 1000):
        assert T > 1 << 30 or call(*_changed(base, T=T, **changes)) == EINVAL, T
    if not torch.cuda.device_count():  # (the addresses are made up)
        for T in (most - 1000, most):
            assert call(*_changed(base, T=T, **changes)) == EUNSUPPORTED, T


def test_workspace_sizes(lib):
    size = lib.mx_attention_kv_workspace
    assert size(0, 0, 8, 2, 128) == 0 and size(3, 0, 8, 2, 128) == 0
    assert size(1, 1, 8, 2, 128) > 0 and size(64, 64, 64, 8, 128) < 1 << 28
    assert size(1, 1, 8, 3, 128) == EINVAL and size(-1, 1, 8, 2, 128) == EINVAL and size(1, 1, 8, 2, 100) == EUNSUPPORTED


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("S, new, many", [(1, 32, False), (1, 64, True), (1, 512, True), (16, 8, False), (16, 16, False), (16, 32, True), (8, 32, False), (64, 16, True)])
def test_the_kernel_for_a_size_is_the_same_for_all_heads(lib, D, S, new, many):
    """Which kernel a call takes, seen from the workspace that it asks for: by rows and key heads, at every head size where it was measured."""
    size = (S, S * new, 64, 8, D)
    few_rows, many_rows = (lib.mx_internal_attention_kv_workspace(force, *size) for force in (1, 2))
    assert lib.mx_attention_kv_workspace(*size) == (many_rows if many else few_rows)


def test_binding_refuses_what_is_not_on_the_gpu():
    torch = pytest.importorskip("torch")
    import paper_2603_08713_amd as mx

    k_cache, v_cache = mx.mx_kv_cache(2, 2, 128, 16, device="cpu")
    assert k_cache[0].shape == (2, 2, 4, 16, 16) and v_cache[0].shape == (2, 2, 4, 16, 4, 4) and k_cache[2].shape == (2, 2, 1, 16)
    assert mx.mx_kv_cache(1, 1, 64, 16, use_mbs=False, device="cpu")[1][2] is None
    x = torch.zeros((1, 2, 128), dtype=torch.bfloat16)
    i64, i32 = torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        mx.mx_kv_write(x, x, i64[:1], k_cache, v_cache)
    with pytest.raises(TypeError):
        mx.mx_kv_read(i64[:1], k_cache, v_cache)
    with pytest.raises(TypeError):
        mx.mx_qk_norm_rope(x, x, i32, torch.zeros((4, 128)))
    with pytest.raises(TypeError):
        mx.mx_attention_kv(x, i64, i32, torch.zeros((1, 1), dtype=torch.int32), k_cache, v_cache)
    with pytest.raises(TypeError):
        mx.mx_kv_plan(i32, i32, 16, torch.zeros((1, 1), dtype=torch.int32), i32, i32, 1)
