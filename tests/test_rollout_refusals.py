"""What the calls around the verify step refuse on the host, before anything touches a GPU: each argument on its own."""
import ctypes

import pytest
import torch

from paper_2510_26475_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
PTR = ctypes.c_void_p(0x100000)      # (never followed: every call here is refused)
ODD = ctypes.c_void_p(0x100001)
BF16, F32 = binding.RESPEC_BF16, binding.RESPEC_F32

CALLS = {
    "respec_prompt_attention": dict(
        q=PTR, k=PTR, v=PTR, q_indptr=PTR, kv_indptr=PTR, out=PTR, lse=None, B=2, total_q=100, total_kv=200, max_q=60, max_kv=120, Hq=8,
        Hkv=2, D=128, ld_q=1024, ld_k=256, ld_v=256, sm_scale=0.1, dt=BF16, workspace=PTR, workspace_bytes=1 << 30, stream=None),
    "respec_prompt_attention_paged": dict(
        q=PTR, k_pages=PTR, v_pages=PTR, q_indptr=PTR, page_indptr=PTR, page_table=PTR, kv_len=PTR, out=PTR, lse=None, B=2, total_q=100,
        num_pages=20, page_table_len=20, page_size=16, max_q=60, max_kv=120, Hq=8, Hkv=2, D=128, ld_q=1024, sm_scale=0.1, dt=BF16,
        workspace=PTR, workspace_bytes=1 << 30, stream=None),
    "respec_append_paged": dict(
        k_new=PTR, v_new=PTR, k_pages=PTR, v_pages=PTR, q_indptr=PTR, page_indptr=PTR, page_table=PTR, kv_len=PTR, B=2, total_q=100, max_q=60,
        num_pages=20, page_table_len=20, page_size=16, Hkv=2, D=128, ld_new=256, dt=BF16, stream=None),
    "respec_pages_resize": dict(
        want=PTR, page_indptr=PTR, page_table=PTR, page_count=PTR, kv_len=PTR, page_refs=PTR, copy_src=PTR, copy_dst=PTR, missing=PTR, B=4,
        page_table_len=40, num_pages=30, page_size=16, workspace=PTR, workspace_bytes=1 << 20, stream=None),
    "respec_pages_fork": dict(
        parent=PTR, page_indptr=PTR, page_table=PTR, page_count=PTR, kv_len=PTR, page_refs=PTR, missing=PTR, B=4, page_table_len=40,
        num_pages=30, stream=None),
    "respec_pages_compact": dict(
        page_table=PTR, page_refs=PTR, new_table=PTR, new_refs=PTR, copy_src=PTR, copy_dst=PTR, end=PTR, page_table_len=40, num_pages=30,
        max_moves=5, workspace=PTR, workspace_bytes=1 << 20, stream=None),
    "respec_pages_copy": dict(
        k_pages=PTR, v_pages=PTR, copy_src=PTR, copy_dst=PTR, n=5, num_pages=30, page_size=16, Hkv=2, D=128, dt=BF16, stream=None),
    "respec_token_logprobs": dict(
        logits=PTR, tokens=PTR, row_T=None, logprob=PTR, lse=PTR, entropy=None, top_tokens=PTR, top_logprobs=PTR, rows=4, V=1000, ld=1000,
        top=5, T=1.0, dt=BF16, workspace=PTR, workspace_bytes=1 << 30, stream=None),
    "respec_token_logprobs_grad": dict(
        logits=PTR, tokens=PTR, row_T=None, lse=PTR, entropy=PTR, g=PTR, h=PTR, grad=PTR, rows=4, V=1000, ld=1000, ld_g=1000, T=1.0, dt=BF16,
        stream=None),
}

MAY_BE_NULL = {"lse": ("respec_prompt_attention", "respec_prompt_attention_paged"), "entropy": ("respec_token_logprobs",),
               "g": ("respec_token_logprobs_grad",), "h": ("respec_token_logprobs_grad",)}

BAD = [
    ("respec_prompt_attention", dict(B=0), INVALID), ("respec_prompt_attention", dict(total_q=0), INVALID),
    ("respec_prompt_attention", dict(total_kv=0), INVALID), ("respec_prompt_attention", dict(max_q=0), INVALID),
    ("respec_prompt_attention", dict(max_kv=-1), INVALID), ("respec_prompt_attention", dict(Hkv=3), INVALID),
    ("respec_prompt_attention", dict(D=96), UNSUPPORTED), ("respec_prompt_attention", dict(dt=2), INVALID),
    ("respec_prompt_attention", dict(sm_scale=float("nan")), INVALID), ("respec_prompt_attention", dict(ld_q=1023), INVALID),
    ("respec_prompt_attention", dict(ld_k=255), INVALID), ("respec_prompt_attention", dict(ld_v=257), UNSUPPORTED),
    ("respec_prompt_attention", dict(q=ODD), INVALID), ("respec_prompt_attention", dict(out=ODD), INVALID),
    ("respec_prompt_attention", dict(workspace=ctypes.c_void_p(0x100010)), WORKSPACE),
    ("respec_prompt_attention", dict(workspace_bytes=10), WORKSPACE), ("respec_prompt_attention", dict(workspace=None), WORKSPACE),
    ("respec_prompt_attention", dict(total_q=1 << 30, max_q=1 << 30, B=1, max_kv=1 << 30), UNSUPPORTED),
    ("respec_prompt_attention", dict(total_q=1 << 24, max_q=1, B=1 << 24, max_kv=1), UNSUPPORTED),
    ("respec_prompt_attention", dict(max_kv=2 ** 31 - 200), UNSUPPORTED),
    ("respec_append_paged", dict(B=1 << 24, total_q=1 << 24, max_q=1), UNSUPPORTED), ("respec_pages_fork", dict(B=1 << 24), UNSUPPORTED),
    ("respec_token_logprobs", dict(rows=1 << 24), UNSUPPORTED), ("respec_token_logprobs_grad", dict(rows=1 << 24), UNSUPPORTED),
    ("respec_prompt_attention_paged", dict(page_size=24), UNSUPPORTED), ("respec_prompt_attention_paged", dict(page_size=8), UNSUPPORTED),
    ("respec_prompt_attention_paged", dict(num_pages=0), INVALID), ("respec_prompt_attention_paged", dict(page_table_len=0), INVALID),
    ("respec_prompt_attention_paged", dict(workspace_bytes=0), WORKSPACE), ("respec_prompt_attention_paged", dict(ld_q=1028), UNSUPPORTED),
    ("respec_append_paged", dict(total_q=0), INVALID), ("respec_append_paged", dict(ld_new=255), INVALID),
    ("respec_append_paged", dict(ld_new=257), UNSUPPORTED), ("respec_append_paged", dict(D=3), UNSUPPORTED),
    ("respec_append_paged", dict(k_new=ODD), INVALID), ("respec_append_paged", dict(page_size=2048), UNSUPPORTED),
    ("respec_append_paged", dict(dt=7), INVALID),
    ("respec_pages_resize", dict(B=0), INVALID), ("respec_pages_resize", dict(num_pages=0), INVALID),
    ("respec_pages_resize", dict(page_size=48), UNSUPPORTED), ("respec_pages_resize", dict(workspace_bytes=100), WORKSPACE),
    ("respec_pages_resize", dict(page_table_len=(1 << 30) - 2), UNSUPPORTED),
    ("respec_pages_fork", dict(page_table_len=0), INVALID), ("respec_pages_fork", dict(B=-3), INVALID),
    ("respec_pages_compact", dict(max_moves=0), INVALID), ("respec_pages_compact", dict(num_pages=-1), INVALID),
    ("respec_pages_compact", dict(workspace=None), WORKSPACE),
    ("respec_pages_copy", dict(n=0), INVALID), ("respec_pages_copy", dict(D=4, Hkv=1), UNSUPPORTED),
    ("respec_pages_copy", dict(k_pages=ODD), INVALID), ("respec_pages_copy", dict(page_size=17), UNSUPPORTED),
    ("respec_token_logprobs", dict(rows=0), INVALID), ("respec_token_logprobs", dict(V=0), INVALID),
    ("respec_token_logprobs", dict(ld=999), INVALID), ("respec_token_logprobs", dict(T=0.0), INVALID),
    ("respec_token_logprobs", dict(T=float("inf")), INVALID), ("respec_token_logprobs", dict(T=1e-40), INVALID),
    ("respec_token_logprobs", dict(top=-1), INVALID), ("respec_token_logprobs", dict(top=65), UNSUPPORTED),
    ("respec_token_logprobs", dict(top_tokens=None), INVALID), ("respec_token_logprobs", dict(logits=ODD), INVALID),
    ("respec_token_logprobs", dict(workspace_bytes=64), WORKSPACE), ("respec_token_logprobs", dict(dt=-1), INVALID),
    ("respec_token_logprobs_grad", dict(g=None, h=None), INVALID), ("respec_token_logprobs_grad", dict(entropy=None), INVALID),
    ("respec_token_logprobs_grad", dict(ld_g=10), INVALID), ("respec_token_logprobs_grad", dict(T=-1.0), INVALID),
    ("respec_token_logprobs_grad", dict(grad=ODD), INVALID), ("respec_token_logprobs_grad", dict(rows=1 << 30, V=1 << 20, ld=1 << 20, ld_g=1 << 20), UNSUPPORTED),
]


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
    f = binding.respec_prompt_attention_workspace_bytes
    assert f(4, 1000, 1000, 400, 400, 28, 4, 128, BF16) >= 256
    assert f(1, 40, 9000, 40, 9000, 28, 4, 128, BF16) > 256        # few rows over many keys: parts
    for bad in ((0, 1000, 1000, 400, 400, 28, 4, 128, BF16), (4, 1000, 0, 400, 400, 28, 4, 128, BF16),
                (4, 1000, 1000, 400, 400, 28, 5, 128, BF16), (4, 1000, 1000, 400, 400, 28, 4, 96, BF16), (4, 1000, 1000, 400, 400, 28, 4, 128, 3)):
        assert f(*bad) == 0
    assert binding.respec_pages_workspace_bytes(0, 5) == binding.respec_pages_workspace_bytes(5, 0) == 0
    assert binding.respec_pages_workspace_bytes(300, 100000) >= 4 * 100600
    assert binding.respec_token_logprobs_workspace_bytes(1, 5, 65, F32) == 0 == binding.respec_token_logprobs_workspace_bytes(0, 5, 5, F32)
    assert len({binding.respec_token_logprobs_workspace_bytes(r, V, 5, F32) for r in (1, 9, 5000) for V in (3, 151936)}) == 1


def test_the_binding_wants_tensors_of_the_current_gpu():
    x, i = torch.zeros((2, 8)), torch.zeros(2, dtype=torch.int32)
    f = torch.zeros(2)
    with pytest.raises(ValueError, match="GPU"):
        binding.respec_token_logprobs(x, i, f, f, None, None, None, 1.0, None)
    with pytest.raises(ValueError, match="GPU"):
        binding.respec_pages_fork(i, torch.zeros(3, dtype=torch.int32), i, i, i, i, i)
