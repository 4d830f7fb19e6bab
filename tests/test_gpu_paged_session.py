"""Rows that rotate makes, in the framework's own decode steps and over bf16 pages: the same step of a multimodal model, an ordinary layer and a lazy one."""

import math

import numpy as np
import pytest
import torch

from oracle.lazy_attention import LazyAttentionOracle
from paged_util import DEV, check_rows, gen, rotation, rows
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import paged
from paper_2602_01901_b200.session import Session, bits_of

from parity_util import assert_close, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group", [(128, 1), (128, 4), (64, 3)])
def test_rotated_rows_in_a_session_and_over_pages(d, group):
    g = gen(d + group)
    hkv, page, n, visual, text, steps = 2, 16, 2, 40, 23, 5
    hq, layers = hkv * group, [0, 1]
    rot, freqs, axes = rotation(d, 3, g)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).bfloat16() for _ in "qk")
    turn = dict(q_norm=wq.to(DEV), k_norm=wk.to(DEV), eps=1e-6)
    session = Session(2, hq, hkv, d, layers, max_seqs=n, max_tokens_per_seq=128, n_pages=200, lazy_mode=qc.QC_MODE_VLA_QC, poison_pool=True)
    oracle = LazyAttentionOracle(2, hq, hkv, d, layers, qc.QC_MODE_VLA_QC, n_seqs=n)
    images, texts = paged.PageTable.empty(n, 8, page, 20), paged.PageTable.empty(n, 8, page, 20)
    image_k = paged.empty_pool(hkv, d, page, 20)                         # the lazy layer reads the first one's
    image_v, text_k, text_v = ([paged.empty_pool(hkv, d, page, 20) for _ in layers] for _ in range(3))
    # prompts: an image's patches at rows and columns of their own, then text
    kind = np.array([1] * visual + [0] * text, np.uint8)
    place = torch.cat([torch.stack([torch.zeros(visual), torch.arange(visual) // 8, torch.arange(visual) % 8]), (visual // 8 + torch.arange(text)).expand(3, -1)], 1).to(torch.int32)
    for s in range(n):
        one = torch.tensor([s], dtype=torch.int32, device=DEV)
        _, image_slots = paged.table_extend(images, torch.tensor([visual], dtype=torch.int32, device=DEV), seq_ids=one, max_slots=visual)
        _, text_slots = paged.table_extend(texts, torch.tensor([text], dtype=torch.int32, device=DEV), seq_ids=one, max_slots=text)
        ks, vs = [], []
        for l in layers:
            raw, v = rows(visual + text, hkv, d, g), rows(visual + text, hkv, d, g).to(DEV)
            _, k = paged.rotate(None, raw.to(DEV), place.to(DEV), rot, **turn)
            check_rows(k, raw, place.tolist(), freqs, axes, False, wk.double().numpy(), 1e-6)
            paged.append(None if l else image_k, image_v[l], image_slots, None if l else raw[:visual].to(DEV), v[:visual], positions=None if l else place[:, :visual].contiguous().to(DEV),
                         rotation=None if l else rot, k_norm=None if l else turn["k_norm"])
            paged.append(text_k[l], text_v[l], text_slots, raw[visual:].to(DEV), v[visual:], positions=place[:, visual:].contiguous().to(DEV), rotation=rot, k_norm=turn["k_norm"])
            ks.append(k)
            vs.append(v)
        session.prefill_append([s], [visual + text], kind, torch.stack(ks), torch.stack(vs))
        oracle.prefill_append(s, kind.tolist(), *(f64(np.stack([bits_of(x) for x in t])) for t in (ks, vs)))
    for step in range(steps):
        at = torch.full((3, n), visual // 8 + text + step, dtype=torch.int32, device=DEV)
        starts, slots = paged.table_extend(texts)
        session.decode_begin(list(range(n)))
        first, seen = None, []
        for l in layers:
            fused = rows(n, hq + 2 * hkv, d, g).to(DEV)
            q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:].contiguous()
            q, k = paged.rotate(q, k, at, rot, **turn)
            out, lse = torch.empty_like(q), torch.empty(n, hq, device=DEV)
            session.decode_layer(l, q, k, v, out, lse)
            q2 = paged.append(text_k[l], text_v[l], slots, fused[:, hq:hq + hkv], v, q=fused[:, :hq], positions=at, rotation=rot, **turn)
            assert torch.equal(q2, q)
            first = q if l == 0 else first
            # each sequence asks about an image of its own
            out2, lse2 = paged.attend(paged.Stream(q, text_k[l], text_v[l], texts.pages, texts.lens), shared=paged.Stream(first, image_k, image_v[l], images.pages, images.lens),
                                      groups=torch.arange(n + 1, dtype=torch.int32, device=DEV), starts=starts, status=texts.state[1:2])
            seen.append((q, k, v, out, lse, out2, lse2))
        texts.check()
        for s in range(n):
            ref, ref_lse = oracle.decode_step(s, *(f64(np.stack([bits_of(x[i][s]) for x in seen])) for i in range(3)))
            for l in layers:
                for out, lse, what in ((seen[l][3], seen[l][4], "session"), (seen[l][5], seen[l][6], "pages")):
                    assert_close(bits_of(out[s]), ref[l], f"{what}: step {step} sequence {s} layer {l}")
                    np.testing.assert_allclose(lse[s].cpu().numpy(), ref_lse[l], atol=2e-3, rtol=0)
    assert session.stats().device_error == 0
    session.close()
