"""What the calls that write, quantise and share the cache refuse on the host, before anything touches a GPU: each argument on its own."""
import ctypes

import pytest
import torch

from paper_2510_26475_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
PTR = ctypes.c_void_p(0x100000)      # (never followed: every call here is refused)
ODD = ctypes.c_void_p(0x100004)
BF16, F32, E4M3 = binding.RESPEC_BF16, binding.RESPEC_F32, binding.RESPEC_E4M3

SHARED = dict(
    q=PTR, k_pages=PTR, v_pages=PTR, k_scale=PTR, v_scale=PTR, q_indptr=PTR, page_indptr=PTR, page_table=PTR, kv_len=PTR, group_indptr=PTR, shared_len=PTR,
    tree_mask=None, out=PTR, lse=None, B=4, total_q=16, groups=2, num_pages=20, page_table_len=20, page_size=16, max_q=4, max_kv=200, Hq=8, Hkv=2, D=128,
    sm_scale=0.1, dt=BF16, pool_dt=E4M3, workspace=PTR, workspace_bytes=1 << 40, stream=None)
CALLS = {
    "respec_norm_rope_append_paged": dict(
        q=PTR, k=PTR, v=PTR, q_weight=PTR, k_weight=PTR, inv_freq=PTR, positions=None, q_out=PTR, k_pages=PTR, v_pages=PTR, k_scale=PTR, v_scale=PTR,
        q_indptr=PTR, page_indptr=PTR, page_table=PTR, kv_len=PTR, B=2, total_q=100, max_q=60, num_pages=20, page_table_len=20, page_size=16, Hq=8, Hkv=2, D=128,
        rotary=64, interleaved=0, ld_q=1024, ld_k=256, ld_v=256, ld_out=1024, eps=1e-6, dt=BF16, pool_dt=E4M3, stream=None),
    "respec_read_paged_quantised": dict(
        k_pages=PTR, v_pages=PTR, k_scale=PTR, v_scale=PTR, page_indptr=PTR, page_table=PTR, kv_len=PTR, kv_indptr=PTR, k_out=PTR, v_out=PTR, B=2, total_kv=100,
        max_kv=60, num_pages=20, page_table_len=20, page_size=16, Hkv=2, D=128, dt=BF16, stream=None),
    "respec_commit_accepted_paged_quantised": dict(
        k_pages=PTR, v_pages=PTR, k_scale=PTR, v_scale=PTR, q_indptr=PTR, page_indptr=PTR, page_table=PTR, kv_len=PTR, path=None, path_stride=0, num_accepted=PTR,
        B=2, total_q=8, max_q=4, num_pages=20, page_table_len=20, page_size=16, Hkv=2, D=128, stream=None),
    "respec_pages_copy_quantised": dict(
        k_pages=PTR, v_pages=PTR, k_scale=PTR, v_scale=PTR, copy_src=PTR, copy_dst=PTR, n=5, num_pages=30, page_size=16, Hkv=2, D=128, stream=None),
    "respec_verify_attention_shared": SHARED,
    "respec_verify_attention_shared_next_layer": SHARED,
    "respec_verify_attention_paged_quantised": {k: v for k, v in SHARED.items() if k not in ("group_indptr", "shared_len", "groups", "pool_dt")},
}
MAY_BE_NULL = {"q_weight": ("respec_norm_rope_append_paged",), "k_weight": ("respec_norm_rope_append_paged",)}

W, R, C, P, S = list(CALLS)[:5]
BAD = [
    (W, dict(B=0), INVALID), (W, dict(total_q=-1), INVALID), (W, dict(max_q=0), INVALID), (W, dict(num_pages=0), INVALID), (W, dict(Hkv=0), INVALID),
    (W, dict(Hq=0), INVALID), (W, dict(q=None), INVALID), (W, dict(q=None, q_out=None), INVALID), (W, dict(dt=E4M3), INVALID), (W, dict(dt=5), INVALID),
    (W, dict(pool_dt=BF16), INVALID), (W, dict(pool_dt=F32, k_scale=None, v_scale=None), INVALID), (W, dict(v_scale=None), INVALID),
    (W, dict(D=96), UNSUPPORTED), (W, dict(rotary=130), INVALID), (W, dict(rotary=-16), INVALID), (W, dict(rotary=0), INVALID), (W, dict(rotary=24), UNSUPPORTED),
    (W, dict(inv_freq=None), INVALID), (W, dict(eps=-1.0), INVALID), (W, dict(eps=float("nan")), INVALID), (W, dict(page_size=24), UNSUPPORTED),
    (W, dict(ld_q=1023), INVALID), (W, dict(ld_k=255), INVALID), (W, dict(ld_v=257), UNSUPPORTED), (W, dict(ld_out=1025), UNSUPPORTED), (W, dict(k=ODD), INVALID),
    (W, dict(q_out=ODD), INVALID), (W, dict(k_weight=ODD), INVALID), (W, dict(v_pages=ODD), INVALID), (W, dict(k_scale=ODD), INVALID), (W, dict(total_q=2 ** 31 - 1), UNSUPPORTED),
    (W, dict(Hq=1 << 17, ld_q=1 << 24, ld_out=1 << 24), UNSUPPORTED),
    (R, dict(B=0), INVALID), (R, dict(total_kv=0), INVALID), (R, dict(max_kv=0), INVALID), (R, dict(dt=E4M3), INVALID), (R, dict(D=32), UNSUPPORTED),
    (R, dict(page_size=8), UNSUPPORTED), (R, dict(k_out=ODD), INVALID), (R, dict(v_scale=ODD), INVALID), (R, dict(total_kv=1 << 40), UNSUPPORTED),
    (C, dict(B=0), INVALID), (C, dict(path=PTR), INVALID), (C, dict(max_q=0), INVALID), (C, dict(B=1 << 24), UNSUPPORTED), (C, dict(k_pages=ODD), INVALID),
    (C, dict(Hkv=1 << 20), UNSUPPORTED), (P, dict(n=0), INVALID), (P, dict(num_pages=0), INVALID), (P, dict(page_size=2048), UNSUPPORTED), (P, dict(D=100), UNSUPPORTED),
]
for name in (S, "respec_verify_attention_shared_next_layer", "respec_verify_attention_paged_quantised"):
    BAD += [(name, a, c) for a, c in (
        (dict(B=0), INVALID), (dict(total_q=0), INVALID), (dict(max_kv=0), INVALID), (dict(Hkv=3), INVALID), (dict(D=80), UNSUPPORTED), (dict(dt=F32), UNSUPPORTED),
        (dict(dt=E4M3), INVALID), (dict(k_scale=None), INVALID), (dict(sm_scale=float("inf")), INVALID), (dict(page_size=40), UNSUPPORTED),
        (dict(total_q=400, max_q=65), UNSUPPORTED), (dict(total_q=70, max_q=65, Hkv=8, tree_mask=PTR), UNSUPPORTED), (dict(B=65536, total_q=65536), UNSUPPORTED),
        (dict(total_q=1 << 28), UNSUPPORTED), (dict(max_kv=2 ** 31 - 200), UNSUPPORTED), (dict(q=ODD), INVALID), (dict(out=ODD), INVALID),
        (dict(k_scale=ODD), INVALID), (dict(v_scale=ODD), INVALID), (dict(workspace=ctypes.c_void_p(0x100010)), WORKSPACE), (dict(workspace_bytes=1000), WORKSPACE))]
BAD += [(S, dict(groups=-1), INVALID), (S, dict(pool_dt=BF16), INVALID), (S, dict(pool_dt=F32, k_scale=None, v_scale=None), INVALID)]


def status(name, **changed):
    lib = binding.load()
    assert set(changed) <= set(CALLS[name])
    return getattr(lib, name)(*{**CALLS[name], **changed}.values()), lib.respec_last_error().decode()


@pytest.mark.parametrize("name,changed,code", BAD, ids=[f"{n[7:]}-{'-'.join(c)}-{i}" for i, (n, c, _) in enumerate(BAD)])
def test_refused(name, changed, code):
    got, text = status(name, **changed)
    assert got == code and text.startswith(name[len("respec_"):])


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_pointers(name):
    for arg, value in CALLS[name].items():
        if value is PTR and name not in MAY_BE_NULL.get(arg, ()):
            got, text = status(name, **{arg: None})
            assert got == (WORKSPACE if arg == "workspace" else INVALID), arg


def test_workspaces():
    f = binding.respec_verify_attention_shared_workspace_bytes
    good = (4, 16, 2, 4, 200, 8, 2, 128, BF16)
    assert f(*good) >= 256
    sizes = [f(B, 4 * B, B // 2, 4, 200, 8, 2, 128, BF16) for B in (1, 2, 5, 100, 1000)]
    assert sizes == sorted(sizes)                                  # one for the largest batch does for every smaller one
    assert f(4, 16, 0, 4, 200, 8, 2, 128, BF16) < f(*good)
    for bad in ((0,) + good[1:], (4, 0) + good[2:], good[:2] + (-1,) + good[3:], good[:6] + (3, 128, BF16), good[:7] + (96, BF16), good[:8] + (E4M3,), (4, 300, 2, 65) + good[4:]):
        assert f(*bad) == 0


def test_the_binding_checks_tensors():
    i, x = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 1, 64))
    pool, codes = torch.zeros((1, 16, 1, 64)), torch.zeros((1, 16, 1, 64), dtype=torch.uint8)
    scale = torch.zeros((1, 1, 16), dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        binding.respec_norm_rope_append_paged(None, x, x, None, None, None, None, None, pool, pool, None, None, i, i, i, i[:1], 1, 0.0)
    with pytest.raises(TypeError, match="e4m3"):
        binding.respec_norm_rope_append_paged(None, x, x, None, None, None, None, None, pool, pool, scale, scale, i, i, i, i[:1], 1, 0.0)
    with pytest.raises(ValueError, match="v_scale"):
        binding.respec_pages_copy_quantised(codes, codes, scale, scale.transpose(1, 2), i, i)
    with pytest.raises(ValueError, match="k_scale and v_scale"):
        binding.respec_pages_copy_quantised(codes, codes, None, None, i, i)
    with pytest.raises(ValueError, match="GPU"):
        binding.respec_verify_attention_shared(x, codes, codes, scale, scale, i, i, i, i[:1], None, None, None, x, None, 1, 16, 0.1, None)
