"""Refusals of the prompt-side calls, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2603_14224_amd as sik

F = 256 * 1000  # never dereferenced: validation fails first
P = ctypes.pointer


def L(**kw):
    base = dict(batch=2, n_kv_heads=2, n_q_heads=8, head_dim=128, max_len=4096, kv_dtype=sik.SIK_BF16)
    base.update(kw)
    return sik.make_layout(**base)


def chunk(**kw):
    return sik.Chunk(**{**dict(n=16, seq_len=F), **kw})


BAD_PAGES = [(dict(page_table=None), -1), (dict(page_len=8), -2), (dict(page_len=48), -2), (dict(page_len=0), -2),
             (dict(n_pages=0), -2), (dict(pages_per_seq=0), -2), (dict(pages_per_seq=63), -2), (dict(page_len=-64), -2)]


def pages(**kw):
    return P(sik.Pages(**{**dict(page_table=F, pages_per_seq=64, page_len=64, n_pages=10), **kw}))


def test_every_call_checks_layout_chunk_and_pages():
    lib = sik.lib()
    rope = sik.RopeArgs(q=F, k=F + 256, v=F, q_out=F + 512, K=F, V=F + 256)
    ev = dict(mass=F, seq_len=F, n_keep=8, keep=F, workspace=F, workspace_bytes=1 << 40)

    def calls(lay, ch):
        lay = None if lay is None else P(lay)
        ch = None if ch is None else P(ch)
        return [lib.sik_rope_append(lay, ch, P(rope)), lib.sik_chunk_attn(lay, ch, F, F, F, 0.0, F + 256, None, F, 1 << 40, None),
                lib.sik_attn_mass(lay, ch, F, F, 0.0, F, 1, None, F, None)]

    assert calls(None, chunk()) == [-1] * 3 and calls(L(), None) == [-1] * 3
    assert calls(L(head_dim=64), chunk()) == [-2] * 3
    assert calls(L(kv_dtype=2), chunk()) == [-3] * 3
    assert calls(L(), chunk(seq_len=None)) == [-1] * 3
    assert calls(L(), chunk(n=0)) == [-5] * 3 and calls(L(), chunk(n=4097)) == [-5] * 3
    for bad, status in BAD_PAGES:
        assert calls(L(), chunk(pages=pages(**bad))) == [status] * 3
        assert lib.sik_evict(P(L()), P(sik.EvictArgs(**ev, pages=pages(**bad)))) == status
    assert lib.sik_evict(None, P(sik.EvictArgs(**ev))) == -1 and lib.sik_evict(P(L()), None) == -1
    assert lib.sik_evict(P(L(head_dim=64)), P(sik.EvictArgs(**ev))) == -2


def test_rope_refusals():
    def call(lay=None, **kw):
        a = dict(q=F, k=F + 256, v=F + 512, q_out=F + 1024, K=F + 2048, V=F + 4096, inv_freq=F, rotary_dim=128, eps=1e-6)
        a.update(kw)
        return sik.lib().sik_rope_append(P(L()), P(chunk()), P(sik.RopeArgs(**a)))

    for name in ("q", "k", "v", "q_out", "K", "V", "inv_freq"):
        assert call(**{name: None}) == -1
    assert call(k_out=F) == -1 and call(k_out=F, K=None, V=None) == -1  # keys go to one place, values only into a cache
    assert call(interleaved=2) == -8 and call(eps=-1.0) == -8 and call(eps=float("nan")) == -8
    for r in (-16, 8, 100, 144):
        assert call(rotary_dim=r) == -2
    assert call(q_stride=1000) == -2 and call(k_stride=255) == -2 and call(v_stride=248) == -2
    assert call(q_stride=1025) == -10 and call(v_stride=260) == -10 and call(k_stride=264 + 4) == -10
    for name in ("q", "k", "v", "q_out", "K", "V", "q_weight", "k_weight"):
        assert call(**{name: F + 8}) == -10
    assert call(q_out=F) == -8 and call(q_out=F + 256) == -8 and call(V=F + 2048) == -8
    assert call(v=None, K=None, V=None, k_out=F + 256) == -8 and call(v=None, K=None, V=None, k_out=F + 1024) == -8


def test_attention_and_weight_refusals():
    lib, lay, ch = sik.lib(), P(L()), P(chunk())
    size = sik.sik_chunk_workspace_bytes(L(), 16)
    good = dict(q=F, K=F, V=F, out=F + 256, lse=None, ws=F, n=size)

    def attn(**kw):
        a = {**good, **kw}
        return lib.sik_chunk_attn(lay, ch, a["q"], a["K"], a["V"], 0.0, a["out"], a["lse"], a["ws"], a["n"], None)

    for name in ("q", "K", "V", "out"):
        assert attn(**{name: None}) == -1 and attn(**{name: F + 4}) == -10
    assert attn(out=F) == -8
    assert attn(ws=None) == -6 and attn(ws=F + 16) == -6 and attn(n=size - 1) == -6
    assert lib.sik_attn_mass(lay, ch, None, F, 0.0, F, 1, None, F, None) == -1
    assert lib.sik_attn_mass(lay, ch, F, F, 0.0, None, 1, None, F, None) == -1
    assert lib.sik_attn_mass(lay, ch, F, F, 0.0, F, 1, None, None, None) == -1
    assert lib.sik_attn_mass(lay, ch, F, F + 2, 0.0, F, 1, None, F, None) == -10
    for n_obs in (0, -1, 17):
        assert lib.sik_attn_mass(lay, ch, F, F, 0.0, F, n_obs, None, F, None) == -5


def test_evict_refusals():
    size = sik.sik_chunk_workspace_bytes(L(), 1)

    def call(**kw):
        a = dict(mass=F, seq_len=F, n_keep=64, keep=F, K=F, V=F + 256, K_out=F + 512, V_out=F + 1024, out_len=64, workspace=F,
                 workspace_bytes=size)
        a.update(kw)
        return sik.lib().sik_evict(P(L()), P(sik.EvictArgs(**a)))

    for name in ("mass", "seq_len", "keep", "K", "V", "K_out", "V_out"):
        assert call(**{name: None}) == -1
    assert call(n_keep=0) == -4 and call(n_keep=4097) == -4
    assert call(n_sink=-1) == -4 and call(n_recent=-1) == -4 and call(n_sink=40, n_recent=25) == -4
    assert call(n_sink=2**31 - 1, n_recent=2**31 - 1) == -4
    assert call(out_len=63) == -5 and call(K_out=None, V_out=None, mass_out=F + 256, out_len=63) == -5
    assert call(K_out=F) == -8 and call(V_out=F + 256) == -8 and call(V_out=F + 512) == -8 and call(mass_out=F) == -8
    assert call(K=F + 8) == -10 and call(V_out=F + 1032) == -10
    assert call(workspace=None) == -6 and call(workspace_bytes=size - 1) == -6


def test_workspace_bytes():
    assert sik.sik_chunk_workspace_bytes(L(), 16) > 0 and sik.sik_chunk_workspace_bytes(L(), 16) % 256 == 0
    for lay, n in ((L(head_dim=64), 1), (L(), 0), (L(), 4097), (L(batch=0), 1)):
        assert sik.sik_chunk_workspace_bytes(lay, n) == 0
    # a buffer for chunks of up to n tokens serves the shorter ones
    for lay in (L(), L(batch=1, max_len=131072), L(n_kv_heads=1, n_q_heads=1, max_len=1 << 20)):
        sizes = [sik.sik_chunk_workspace_bytes(lay, n) for n in (1, 2, 3, 7, 8, 9, 16, 33, 100, 257, 1000, 4000)]
        assert sizes == sorted(sizes)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors below are the CPU's")
def test_binding_checks_types_and_shapes():
    lay = L(max_len=64)
    lens = torch.zeros(2, dtype=torch.int32)
    ch = sik.make_chunk(4, lens)
    q, k = torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 2, 128, dtype=torch.bfloat16)
    cache = torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16)
    bad = [dict(q=q.half()), dict(q=q[:, :3]), dict(q=q.transpose(1, 2)), dict(q=torch.zeros(2, 8, 8, 128, dtype=torch.bfloat16)[:, ::2][:, :, :, :]),
           dict(K=cache.half()), dict(K=cache[:, :, :32]), dict(q_weight=torch.zeros(64)),
           dict(inv_freq=torch.zeros(64, dtype=torch.float64)), dict(positions=torch.zeros(2, 4)), dict(q_out=k)]
    bad[3]["q"] = torch.zeros(2, 9, 8, 128, dtype=torch.bfloat16)[:, :8:2]  # evenly spaced tokens, sequences that are not
    for kw in bad:
        a = dict(q=q, q_out=torch.zeros_like(q), K=cache, V=cache.clone(), q_weight=None, inv_freq=None, positions=None)
        a.update(kw)
        with pytest.raises(ValueError):
            sik.sik_rope_append(lay, ch, a["q"], k, a["q_out"], v=k, K=a["K"], V=a["V"], q_weight=a["q_weight"],
                                inv_freq=a["inv_freq"], positions=a["positions"])
    with pytest.raises(ValueError):
        sik.make_chunk(4, lens.long())
    with pytest.raises(ValueError):
        sik.sik_attn_mass(lay, sik.make_chunk(4, lens[:1]), q, cache, 0.0, torch.zeros(2, 4, 8), 1, None, torch.zeros(2, 2, 64))
    with pytest.raises(ValueError):
        sik.sik_attn_mass(lay, ch, q, cache, 0.0, torch.zeros(2, 4, 8), 1, None, torch.zeros(2, 2, 63))
    table = torch.zeros(3, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        sik.sik_evict(lay, torch.zeros(2, 2, 64), lens, 8, torch.zeros(2, 2, 8, dtype=torch.int32), None,
                      pages=sik.make_pages(table, 16, 4))
    with pytest.raises(ValueError):
        sik.sik_evict(lay, torch.zeros(2, 2, 64), lens, 8, torch.zeros(2, 2, 9, dtype=torch.int32), None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors below are the CPU's")
@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("B,n,own", [(1, 4, (1, 1)), (3, 1, (1, 1)), (3, 4, (1, 1)), (3, 4, (3, 1)), (3, 4, (1, 4))])
def test_broadcast_rows_are_refused(name, B, n, own):
    # one row for several tokens or sequences: a stride of 0, which to the C side means packed rows, of which there are more
    lay, heads = L(batch=B, max_len=64), dict(q=8, k=2, v=2)
    a = {x: torch.zeros(B, n, h, 128, dtype=torch.bfloat16) for x, h in heads.items()}
    a[name] = torch.zeros(*own, heads[name], 128, dtype=torch.bfloat16).expand(B, n, -1, -1)
    K, V = (torch.zeros(B, 2, 64, 128, dtype=torch.bfloat16) for _ in range(2))
    chunk = sik.make_chunk(n, torch.zeros(B, dtype=torch.int32))
    with pytest.raises(ValueError, match=f"^{name}: "):
        sik.sik_rope_append(lay, chunk, a["q"], a["k"], torch.zeros_like(a["q"], memory_format=torch.contiguous_format),
                            v=a["v"], K=K, V=V)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors below are the CPU's")
def test_overlapping_tokens_are_refused():
    lay = L(batch=1, max_len=64)
    k = torch.zeros(1, 4, 2, 128, dtype=torch.bfloat16)
    q = torch.zeros(4096, dtype=torch.bfloat16).as_strided((1, 4, 8, 128), (4096, 512, 128, 1))
    with pytest.raises(ValueError, match="^q: "):
        sik.sik_rope_append(lay, sik.make_chunk(4, torch.zeros(1, dtype=torch.int32)), q, k, torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16),
                            k_out=torch.zeros_like(k))


def test_evict_refuses_lists_and_lengths_over_its_inputs():
    # a workgroup may still have to read what another one has overwritten
    lay = L(max_len=64)  # 2 x 2 rows of 64 weights, 1024 bytes; two lengths, 8; lists of 16 tokens, 256
    base, far = 256 * 1000, 256 * 2000

    def call(**kw):
        a = dict(mass=base, seq_len=far, new_len=far + 1024, keep=far + 4096, n_keep=16, workspace=far * 2, workspace_bytes=1 << 40)
        a.update(kw)
        return sik.lib().sik_evict(P(lay), P(sik.EvictArgs(**a)))

    for at in (far, far + 4, far - 4):
        assert call(new_len=at) == -8
    for at in (base, base + 1020, base - 4):
        assert call(new_len=at) == -8
    for at in (far, far + 4, far - 252, base, base + 1020, base - 252, far + 1024, far + 1028, far + 1024 - 252):
        assert call(keep=at) == -8
    if not torch.cuda.is_available():  # beside each other: as far as the launch, for which there is no device
        assert call(new_len=far + 8, keep=far + 16) == -7 and call(new_len=base + 1024, keep=base - 256) == -7
