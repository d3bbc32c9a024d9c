"""A layer's prompt, chunk by chunk, and its first decode step (GPU).

Two sequences are prefilled in two chunks each: the chunk's latents and keys
are normalized, rotated and written to the cache; the prefix and the chunk are
read back as dense rows and expanded by the layer's products; the rotated
queries attend over them.  Every chunk's attention equals the 64-bit formula on
the same expanded rows.  The last chunk ends with the token that the absorbed
decode then answers over the cache itself: its lse and its value-projected
output agree with the expanded form's within the roundings that lie between
the two forms.
"""
import math

import numpy as np
import pytest

from prefill_ref import U16, Attended, rotation_table

pytestmark = pytest.mark.gpu

TAU = 1.0 / math.sqrt(192.0)
H, PAGE = 16, 64


@pytest.mark.parametrize("kind", ["bf16", "c4", "c4_prot", "c2_paper"])
def test_chunked_prompt_then_decode(kind):
    import torch

    from paper_2609_36760_amd import _binding as mb
    from paper_2609_36760_amd import _prefill as mp
    from oracle import protection as op
    lens, cuts = [331, 150], [(200, 70), (331, 150)]
    B = len(lens)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def ints(a, t=np.int32):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=t)).cuda()

    bf16, prot = kind == "bf16", kind == "c4_prot"
    fmt = mb.cache_format(c_bits=2 if kind == "c2_paper" else 4, page_size=PAGE,
                          meta=mb.MLA_META_PAPER if kind == "c2_paper" else mb.MLA_META_FP16)
    pages = [-(-n // PAGE) for n in lens]
    table = np.zeros((B, max(pages)), np.int32)
    ids = np.random.default_rng(1).permutation(sum(pages))
    for b, at in enumerate(np.cumsum([0] + pages[:-1])):
        table[b, :pages[b]] = ids[at:at + pages[b]]
    page_bytes = mb.mla_bf16_page_bytes(fmt) if bf16 else mb.mla_lowbit_page_bytes(fmt)
    cache = torch.zeros(sum(pages) * page_bytes, dtype=torch.uint8, device="cuda")
    policy = mb.protect_policy(4, 128)
    buffers = torch.zeros(B * 132 * 576, dtype=torch.bfloat16, device="cuda")
    prot_slot = ints([1, 0])
    x = [normal(n, 512).bfloat16() for n in lens]
    raw_k = [(2.0 * normal(n, 64)).bfloat16() for n in lens]
    q = [normal(n, H, 192).bfloat16() for n in lens]
    w_uk = (normal(512, H, 128) / math.sqrt(512)).bfloat16()
    w_uv = (normal(512, H, 128) / math.sqrt(512)).bfloat16()
    w = torch.cat([w_uk, w_uv], dim=2).reshape(512, H * 256)
    rot, norm = mp.rotation(rotation_table(400).cuda()), mp.rms_norm(1e-6, (1.0 + 0.1 * normal(512)).bfloat16())
    d_table = ints(table)

    done = [0] * B
    for cut in cuts:
        new = [c - d for c, d in zip(cut, done)]
        seq = np.repeat(np.arange(B), new)
        pos = np.concatenate([np.arange(d, c) for d, c in zip(done, cut)])
        slots = table[seq, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
        xs = torch.cat([t[d:c] for t, d, c in zip(x, done, cut)])
        ks = torch.cat([t[d:c] for t, d, c in zip(raw_k, done, cut)])
        c_new, k_new = torch.empty_like(xs), torch.empty_like(ks)
        args = (norm, rot, xs, ks, ints(pos), ints(slots, np.int64), cache, sum(pages))
        if prot:
            mp.mla_lowbit_norm_rope_append_protected(fmt, policy, *args, ints(seq), ints(cut), prot_slot, buffers, B, c_new, k_new)
        elif bf16:
            mp.mla_bf16_norm_rope_append(fmt, *args, c_new, k_new)
        else:
            mp.mla_lowbit_norm_rope_append(fmt, *args, c_new, k_new)
        qs = torch.cat([t[d:c] for t, d, c in zip(q, done, cut)])
        mp.mla_rope_queries(rot, qs[..., 128:], ints(pos))              # in place
        # the prefix and the chunk as the cache holds them
        total = sum(cut)
        cu = ints(np.concatenate([[0], np.cumsum(cut)]))
        c_all = torch.empty((total, 512), dtype=torch.bfloat16, device="cuda")
        k_all = torch.empty((total, 64), dtype=torch.bfloat16, device="cuda")
        if prot:
            mp.mla_lowbit_gather_protected(fmt, policy, cache, sum(pages), d_table, cu, ints(cut), buffers, B, prot_slot, c_all, k_all)
        else:
            (mp.mla_bf16_gather if bf16 else mp.mla_lowbit_gather)(fmt, cache, sum(pages), d_table, cu, c_all, k_all)
        kv = torch.mm(c_all, w).reshape(total, H, 256)
        plan, info = mp.mla_plan_prefill(new, list(cut), H)
        work = torch.empty(info.workspace_bytes, dtype=torch.uint8, device="cuda")
        out, lse = torch.empty((sum(new), H, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((sum(new), H), device="cuda")
        mp.mla_prefill_attn(info, ints(plan), qs[..., :128], qs[..., 128:], kv[..., :128], k_all, kv[..., 128:], TAU, out, lse, work)
        torch.cuda.synchronize()
        a = e = 0
        for b in range(B):
            nq, nk = new[b], cut[b]
            if bf16:        # what was appended is what is read back
                assert torch.equal(c_all[e + done[b]:e + nk], c_new[a:a + nq]) and torch.equal(k_all[e + done[b]:e + nk], k_new[a:a + nq])
            if prot:
                held = op.protected_positions(nk)
                held = held[held >= done[b]]
                rows = torch.from_numpy(held).cuda()
                assert torch.equal(c_all[e + rows], c_new[a + rows - done[b]])
            Attended(qs[a:a + nq, :, :128], qs[a:a + nq, :, 128:], kv[e:e + nk, :, :128], k_all[e:e + nk], kv[e:e + nk, :, 128:],
                     True, TAU).check(out[a:a + nq], lse[a:a + nq], f"{kind}, {cut}, sequence {b}")
            a, e = a + nq, e + nk
        last_q = [sum(new[:b + 1]) - 1 for b in range(B)]
        done = list(cut)

    # the last token again, absorbed, over the cache
    q_last = qs[last_q]                                                  # [B, H, 192], rotated
    q_lat = torch.stack([torch.mm(q_last[:, h, :128].float(), w_uk[:, h].float().T.contiguous()) for h in range(H)], dim=1)
    q_lat16 = q_lat.bfloat16().reshape(B, 1, H, 512).contiguous()
    q_rope16 = q_last[..., 128:].reshape(B, 1, H, 64).contiguous()
    o_lat, l2 = torch.empty((B, 1, H, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((B, 1, H), device="cuda")
    if prot:
        mb.mla_lowbit_decode_attn_protected(fmt, policy, q_lat16, q_rope16, cache, sum(pages), d_table, ints(lens), 1, H, TAU,
                                            buffers, B, prot_slot, out=o_lat, lse=l2)
    else:
        fn = mb.mla_bf16_decode_attn if bf16 else mb.mla_lowbit_decode_attn
        fn(fmt, q_lat16, q_rope16, cache, sum(pages), d_table, ints(lens), 1, H, TAU, out=o_lat, lse=l2)
    torch.cuda.synchronize()
    e = 0
    for b in range(B):
        nk = lens[b]
        c, kr, exp = c_all[e:e + nk].double(), k_all[e:e + nk].double(), kv[e:e + nk].double()
        for h in range(H):
            qn, qr, ql = q_last[b, h, :128].double(), q_last[b, h, 128:].double(), q_lat[b, h].double()
            # between the forms: k_nope rounded to bf16; q_lat rounded to bf16; the stored latents and keys read as
            # bf16 here and as fp16 (half a step 2^-11) there, scales too; fp32 sums (2^-14 covers them)
            dz = TAU * ((U16 + 2.0 ** -14) * (exp[:, h, :128].abs() @ qn.abs()) + 2.1 * U16 * (c.abs() @ ql.abs())
                        + 1.2 * U16 * (kr.abs() @ qr.abs()))
            dz = float(dz.max())
            got, want = float(l2[b, 0, h]), float(lse[last_q[b], h])
            # (the decode's lse sums rounded weights: at most 2^-8)
            assert abs(got - want) <= 2.0 * dz + U16, (kind, b, h, got, want, dz)
            z = TAU * (exp[:, h, :128] @ qn + kr @ qr)
            wgt = torch.softmax(z, 0)
            v = exp[:, h, 128:]
            mine, other = out[last_q[b], h].double(), o_lat[b, 0, h].double() @ w_uv[:, h].double()
            spread = wgt @ v.abs()
            latent = (wgt @ c.abs()) @ w_uv[:, h].double().abs()
            # weights by e^(2 dz); expanded: v, weights and output in bf16; absorbed: latents, weights, output latent in bf16
            bound = (math.expm1(4.0 * dz) + 4.0 * U16) * spread + 5.0 * U16 * latent
            assert bool(((mine - other).abs() <= bound).all()), (kind, b, h)
        e += nk
    print(f"  {kind}: chunks and decode agree", flush=True)
