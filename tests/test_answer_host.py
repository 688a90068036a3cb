"""Host checks of the calls that answer from a compacted cache: refusals before any launch (no GPU needed), the descriptors' layout, and
the plain forms the GPU tests compare with."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2407_08454_amd import binding as kb

import answer_ref as ar

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE, TWO = ctypes.c_void_p(4096), ctypes.c_void_p(8192)     # never dereferenced: the calls fail before any launch


def _shape(**kw):
    d = dict(B=4, H_kv=2, G=3, N=5, d=128, dtype=kb.KVM_F16, seq_lens=None)
    d.update(kw)
    return kb.KvmShape(**d)


def _pages(**kw):
    d = dict(K=4096, V=4096, table=4096, n_pages=8, page_size=16, max_pages=4)
    d.update(kw)
    return kb.KvmPages(**d)


def _prefix(**kw):
    d = dict(K=4096, V=4096, lens=None, row_start=None, P=2, capacity=100)
    d.update(kw)
    return kb.KvmPrefix(**d)


def _append(shape=None, pages=None, rot=None, q=ONE, qs=1024, k=ONE, ks=1024, v=ONE, vs=1024, past=ONE, pos=None, q_out=TWO, kv=TWO):
    by = lambda x: None if x is None else ctypes.byref(x)
    return kb.load_library().kvm_paged_append(by(shape or _shape()), by(pages or _pages()), by(rot or kb.KvmRotation(4096, 128, 0)), q, qs,
                                              k, ks, v, vs, past, pos, q_out, kv, None)


def _attn(shape=None, prefix=_prefix(), pages=_pages(), q=ONE, qs=1024, kv=ONE, out=ONE, ws=ONE, nbytes=1 << 40):
    by = lambda x: None if x is None else ctypes.byref(x)
    return kb.load_library().kvm_prefix_attn(by(shape or _shape()), by(prefix), by(pages), q, qs, kv, out, None, ws, nbytes, None)


def _message():
    return kb.load_library().kvm_last_error().decode()


@pytest.mark.parametrize("kw,code,word", [
    (dict(shape=_shape(d=64)), kb.KVM_ERR_UNSUPPORTED, "head dimension"),
    (dict(shape=_shape(dtype=5)), kb.KVM_ERR_UNSUPPORTED, "dtype"),
    (dict(shape=_shape(N=-1)), kb.KVM_ERR_INVALID_ARG, "sizes"),
    (dict(shape=_shape(B=4096, N=4096)), kb.KVM_ERR_UNSUPPORTED, "too many"),
    (dict(shape=_shape(B=1024, N=4096, H_kv=128, G=1)), kb.KVM_ERR_UNSUPPORTED, "too many"),
    (dict(pages=_pages(page_size=24)), kb.KVM_ERR_INVALID_ARG, "power of two"),
    (dict(pages=_pages(page_size=0)), kb.KVM_ERR_INVALID_ARG, "pages"),
    (dict(pages=_pages(page_size=1 << 17)), kb.KVM_ERR_INVALID_ARG, "pages"),
    (dict(pages=_pages(n_pages=-1)), kb.KVM_ERR_INVALID_ARG, "pages"),
    (dict(pages=_pages(max_pages=1 << 20)), kb.KVM_ERR_UNSUPPORTED, "too long"),
    (dict(pages=_pages(K=None)), kb.KVM_ERR_INVALID_ARG, "NULL"),
    (dict(pages=_pages(table=None)), kb.KVM_ERR_INVALID_ARG, "NULL"),
    (dict(pages=_pages(V=4104)), kb.KVM_ERR_INVALID_ARG, "16 bytes"),
    (dict(rot=kb.KvmRotation(4096, 24, 0)), kb.KVM_ERR_UNSUPPORTED, "rot_dim"),
    (dict(rot=kb.KvmRotation(4096, 256, 0)), kb.KVM_ERR_UNSUPPORTED, "rot_dim"),
    (dict(rot=kb.KvmRotation(None, 64, 0)), kb.KVM_ERR_INVALID_ARG, "inv_freq"),
    (dict(k=None), kb.KVM_ERR_INVALID_ARG, "k_new"),
    (dict(v=None), kb.KVM_ERR_INVALID_ARG, "v_new"),
    (dict(q=None), kb.KVM_ERR_INVALID_ARG, "together"),
    (dict(q_out=None), kb.KVM_ERR_INVALID_ARG, "together"),
    (dict(k=ctypes.c_void_p(4104)), kb.KVM_ERR_INVALID_ARG, "16 bytes"),
    (dict(ks=1028), kb.KVM_ERR_INVALID_ARG, "16 bytes"),
    (dict(ks=128), kb.KVM_ERR_INVALID_ARG, "apart"),
    (dict(vs=-1024), kb.KVM_ERR_INVALID_ARG, "apart"),
    (dict(q=TWO, q_out=TWO), kb.KVM_ERR_INVALID_ARG, "contiguous"),
    (dict(past=None), kb.KVM_ERR_INVALID_ARG, "two buffers"),
    (dict(kv=None), kb.KVM_ERR_INVALID_ARG, "two buffers"),
    (dict(kv=ONE), kb.KVM_ERR_INVALID_ARG, "two buffers"),
])
def test_append_refuses(kw, code, word):
    assert _append(**kw) == code and word in _message()


@pytest.mark.parametrize("kw", [dict(shape=_shape(seq_lens=8192)), dict(pos=TWO)])
def test_append_refuses_lengths_that_are_written_over_what_it_reads(kw):
    """kv_lens is written by one workgroup while others still read seq_lens and pos_base."""
    assert _append(**kw) == kb.KVM_ERR_INVALID_ARG and "of its own" in _message()


@pytest.mark.parametrize("kw,code,word", [
    (dict(shape=_shape(d=256)), kb.KVM_ERR_UNSUPPORTED, "head dimension"),
    (dict(shape=_shape(B=4096, N=4096)), kb.KVM_ERR_UNSUPPORTED, "too many"),
    (dict(prefix=None, pages=None), kb.KVM_ERR_INVALID_ARG, "both"),
    (dict(prefix=_prefix(P=3)), kb.KVM_ERR_INVALID_ARG, "row_start"),
    (dict(prefix=_prefix(P=-1)), kb.KVM_ERR_INVALID_ARG, "prefix"),
    (dict(prefix=_prefix(capacity=(1 << 22) + 1)), kb.KVM_ERR_INVALID_ARG, "prefix"),
    (dict(prefix=_prefix(K=None)), kb.KVM_ERR_INVALID_ARG, "NULL"),
    (dict(prefix=_prefix(V=4097)), kb.KVM_ERR_INVALID_ARG, "16 bytes"),
    (dict(pages=_pages(page_size=3)), kb.KVM_ERR_INVALID_ARG, "power of two"),
    (dict(q=None), kb.KVM_ERR_INVALID_ARG, "Q must"),
    (dict(qs=640), kb.KVM_ERR_INVALID_ARG, "apart"),
    (dict(out=None), kb.KVM_ERR_INVALID_ARG, "out"),
    (dict(out=ctypes.c_void_p(4100)), kb.KVM_ERR_INVALID_ARG, "16 bytes"),
    (dict(kv=None), kb.KVM_ERR_INVALID_ARG, "kv_lens"),
    (dict(ws=None), kb.KVM_ERR_WORKSPACE, "workspace"),
    (dict(nbytes=16), kb.KVM_ERR_WORKSPACE, "workspace"),
    (dict(ws=ctypes.c_void_p(4100)), kb.KVM_ERR_INVALID_ARG, "aligned"),
])
def test_attention_refuses(kw, code, word):
    assert _attn(**kw) == code and word in _message()


def test_null_descriptors_and_nothing_to_do():
    lib = kb.load_library()
    sh, pg = _shape(), _pages()
    rot = kb.KvmRotation(4096, 128, 0)
    args = (ONE, 1024, ONE, 1024, ONE, 1024, ONE, None, TWO, TWO, None)
    assert lib.kvm_paged_append(None, ctypes.byref(pg), ctypes.byref(rot), *args) == kb.KVM_ERR_INVALID_ARG
    assert lib.kvm_paged_append(ctypes.byref(sh), None, ctypes.byref(rot), *args) == kb.KVM_ERR_INVALID_ARG
    assert lib.kvm_paged_append(ctypes.byref(sh), ctypes.byref(pg), None, *args) == kb.KVM_ERR_INVALID_ARG
    assert _append(shape=_shape(B=0), q=None, k=None, v=None, past=None, kv=None, q_out=None) == kb.KVM_OK
    assert _append(shape=_shape(B=0), pages=_pages(table=None), q=None, k=None, v=None, past=None, kv=None, q_out=None) == kb.KVM_OK
    assert _attn(shape=_shape(B=0), q=None, out=None, ws=None) == kb.KVM_OK
    assert _attn(shape=_shape(B=0), pages=_pages(table=None), q=None, out=None, ws=None) == kb.KVM_OK
    assert _attn(shape=_shape(N=0), q=None, out=None, ws=None) == kb.KVM_OK
    assert lib.kvm_prefix_attn(None, None, ctypes.byref(pg), ONE, 1024, ONE, ONE, None, ONE, 1 << 30, None) == kb.KVM_ERR_INVALID_ARG
    assert lib.kvm_prefix_attn_workspace_bytes(None, None, ctypes.byref(pg)) == 0
    assert lib.kvm_prefix_attn_workspace_bytes(ctypes.byref(sh), None, None) == 0
    assert lib.kvm_prefix_attn_workspace_bytes(ctypes.byref(sh), None, ctypes.byref(pg)) > 0
    with pytest.raises(kb.KvmError):
        kb.kvm_prefix_attn_workspace_bytes(sh, None, None)


@pytest.mark.parametrize("dtype", [kb.KVM_F32, kb.KVM_F16, kb.KVM_BF16])
@pytest.mark.parametrize("B,N", [(0, 1), (0, 3), (0, 32), (0, 200), (0, 0), (4, 0)])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("sources", ["both", "prefix", "pages", "no table", "row_start"])
def test_workspace_of_batches_without_rows_and_steps_without_tokens(dtype, B, N, G, sources):
    """Such a call has nothing to keep: the least size, whichever kernels a row or a token more would take."""
    prefix = None if sources in ("pages", "no table") else _prefix(row_start=4096 if sources == "row_start" else None)
    pages = None if sources == "prefix" else _pages(table=4096 if B or sources != "no table" else None)
    sizes = dict(dtype=dtype, G=G)
    assert kb.kvm_prefix_attn_workspace_bytes(_shape(B=B, N=N, **sizes), prefix, pages) == 256
    assert kb.kvm_prefix_attn_workspace_bytes(_shape(B=4, N=max(N, 1), **sizes), prefix, _pages()) >= 256
    assert _attn(shape=_shape(B=B, N=N, **sizes), prefix=prefix, pages=pages, q=None, out=None, kv=None, ws=None, nbytes=0) == kb.KVM_OK


def test_descriptors_have_the_layout_of_the_header(tmp_path):
    structs = {"kvm_pages": kb.KvmPages, "kvm_rotation": kb.KvmRotation, "kvm_prefix": kb.KvmPrefix}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "kvm.h"', 'int main(void) {']
    for name, cls in structs.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, cls in structs.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f in cls._fields_:
            assert int(got[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset, f"{name}.{f[0]}"


def test_binding_refuses_tensors_that_are_not_on_the_gpu_or_do_not_fit():
    pool, table = torch.zeros((4, 2, 16, 128)), torch.zeros((3, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        kb.make_pages(pool, pool, table)
    with pytest.raises(ValueError):
        kb.make_pages(pool, pool[:2], table)
    with pytest.raises(ValueError):
        kb.make_pages(pool, pool, table.long())
    with pytest.raises(ValueError):
        kb.make_prefix(pool, pool)
    with pytest.raises(ValueError):
        kb.make_rotation(torch.zeros(64, dtype=torch.float64))
    with pytest.raises(ValueError):
        kb.make_rotation(torch.zeros(64))
    # evenly spaced tokens whose heads are contiguous, nothing else
    stride = lambda t, B, T, H: kb._token_stride("x", t, (B, T, H, 128), torch.float32, t.get_device())
    x = torch.zeros((2, 3, 6, 128))
    assert stride(x, 2, 3, 6) == 768 and stride(x[:, :, 2:4], 2, 3, 2) == 768 and stride(x[:, :1], 2, 1, 6) == 3 * 768
    assert stride(x[:1], 1, 3, 6) == 768 and stride(x[:1, 1:2], 1, 1, 6) == 768
    for bad, shape in ((x.transpose(1, 2), (2, 6, 3)), (x[:, :2], (2, 2, 6)), (x[..., ::2, :], (2, 3, 3)), (x.half(), (2, 3, 6)),
                       (x, (3, 2, 6))):
        with pytest.raises(ValueError):
            stride(bad, *shape)


def test_plain_rotation():
    x = np.random.default_rng(0).standard_normal((5, 128))
    f = 1.0 / 10000.0 ** (np.arange(0, 128, 2) / 128)
    assert np.array_equal(ar.rotate(x, np.zeros(5), f, False), x)
    for inter in (False, True):
        y = ar.rotate(x, np.full(5, 7), f, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        # scores depend on the difference of positions only
        a = (ar.rotate(x, np.full(5, 11), f, inter) * ar.rotate(x[::-1], np.full(5, 4), f, inter)).sum(-1)
        b = (ar.rotate(x, np.full(5, 107), f, inter) * ar.rotate(x[::-1], np.full(5, 100), f, inter)).sum(-1)
        assert np.allclose(a, b)
        assert np.array_equal(ar.rotate(x, np.full(5, 3), f[:16], inter)[:, 32:], x[:, 32:])
    perm = np.concatenate([np.arange(0, 128, 2), np.arange(1, 128, 2)])
    assert np.allclose(ar.rotate(x, np.full(5, 9), f, True)[:, perm], ar.rotate(x[:, perm], np.full(5, 9), f, False))
    quarter = ar.rotate(np.eye(128)[:1], np.ones(1), np.full(64, math.pi / 2), False)
    assert np.allclose(quarter[0, 64], 1.0)


def test_plain_attention():
    """Prefix and tail are one sequence: the same keys all in the prefix, all in the tail, or split."""
    rng = np.random.default_rng(1)
    q, K, V = rng.standard_normal((2, 1, 4, 128)), rng.standard_normal((1, 2, 40, 128)), rng.standard_normal((1, 2, 40, 128))

    def tail(first):
        n = 40 - first
        table, n_pages = ar.scattered_pages(rng, 2, [n, n], 8)
        Kp, Vp = np.full((n_pages, 2, 8, 128), np.nan), np.full((n_pages, 2, 8, 128), np.nan)
        for b in range(2):
            for j in range(n):
                Kp[table[b, j // 8], :, j % 8], Vp[table[b, j // 8], :, j % 8] = K[0, :, first + j], V[0, :, first + j]
        return dict(K=Kp, V=Vp, table=table, kv_lens=[n, n])

    whole, lse, _ = ar.attention(q, 2, None, dict(K=K, V=V, lens=None, row_start=None))
    for first in (0, 13, 40):
        part, lse2, _ = ar.attention(q, 2, None, dict(K=K, V=V, lens=np.full((1, 2), first), row_start=[0, 2]), tail(first))
        assert np.allclose(part, whole) and np.allclose(lse2, lse)
    s = torch.from_numpy(q[:, 0].reshape(2, 2, 2, 128)) @ torch.from_numpy(K[0]).transpose(1, 2)
    want = torch.softmax(s / math.sqrt(128), -1) @ torch.from_numpy(V[0])
    assert np.allclose(whole.reshape(2, 2, 2, 128), want.numpy())
    none, l0, _ = ar.attention(q, 2, [1, 0], dict(K=K, V=V, lens=np.zeros((1, 2)), row_start=[0, 2]))
    assert (none[0] == 0).all() and np.isneginf(l0[0]).all() and np.isnan(none[1]).all()
