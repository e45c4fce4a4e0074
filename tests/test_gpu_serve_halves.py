"""fp16 attention over the cache on the GPU against its own bound (tests/serve_halves.py), for every number of query rows that share
a key/value head: up to 8, 16, 24, 32 rows of a tile and several tiles, both head widths, both code widths."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serve_halves as sh
import serve_reference as ref
from test_gpu_serve import build_sequences, cq, make_cache, normal  # noqa: F401  (cq: the fixture)

pytestmark = pytest.mark.gpu

ROWS = ((1, 1), (1, 8), (3, 4), (1, 16), (5, 4), (3, 8), (7, 4), (4, 8), (9, 8))        # query tokens x heads that share one
SHAPES = [(Lq, G, D, bits) for Lq, G in ROWS for D in (64, 128) for bits in (8, 4)]


@pytest.mark.parametrize("Lq,G,D,bits", SHAPES)
@pytest.mark.parametrize("which", ("query_case", "weight_case"))
def test_both_halves_are_there(cq, which, Lq, G, D, bits):  # noqa: F811
    """A sequence for each query row and two heads with cases of their own, one query token each."""
    R, page = Lq * G, 16
    heads = [getattr(sh, which)(R, D, bits, 10 * R + h) for h in range(2)]
    n = heads[0]["kc"].shape[0]
    pages = -(-n // page)
    pad = pages * page - n
    cache = cq.KVCache.empty(pages, page, 2, D, bits, k_col=torch.from_numpy(np.stack([h["kf"] for h in heads])).cuda(),
                             v_col=torch.from_numpy(np.stack([h["vf"] for h in heads])).cuda())
    for name, codes, scale in (("k", "kc", "ka"), ("v", "vc", "va")):
        c = np.stack([np.pad(h[codes], ((0, pad), (0, 0))) for h in heads], axis=1).reshape(pages, page, 2, D).transpose(0, 2, 1, 3)
        s = np.stack([np.pad(h[scale], (0, pad)) for h in heads], axis=1).reshape(pages, page, 2).transpose(0, 2, 1)
        getattr(cache, name + "_codes").copy_(ref.pack(c, bits))
        getattr(cache, name + "_scale").copy_(torch.from_numpy(s.copy()))
    # all rows see all tokens: they share a head (one query token), or are the same sequence's last token again and again
    q = torch.from_numpy(np.stack([h["q"] for h in heads]).reshape(1, 1, 2 * R, D)).half().cuda()
    lse = torch.empty(1, 1, 2 * R, device="cuda")
    out = cq.kv_attention(q, cache, torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"),
                          scale=heads[0]["scale"], lse=lse)
    for h, case in enumerate(heads):
        at = np.s_[h * R:(h + 1) * R]
        worst = sh.worst(out[0, 0, at].cpu().numpy(), lse[0, 0, at].cpu().numpy(), case)
        assert max(worst) <= 1, worst


@pytest.mark.parametrize("Lq,G,D,bits", SHAPES)
def test_against_64_bits(cq, Lq, G, D, bits):  # noqa: F811
    """Ragged sequences with every query row's own limit, empty ones and rows that see nothing among them."""
    lens, H, page = [400, 0, 1, 17, max(1, Lq - 1), 65, 130], 2, 16 if D == 64 else 48
    table, pages = build_sequences(None, lens, page, Lq)
    cache, codes, scales, cols, _ = make_cache(cq, pages, page, H, D, bits, True, G)
    q = normal((len(lens), Lq, H * G, D), Lq + G, torch.float16, outliers=False)
    lse = torch.empty(len(lens), Lq, H * G, device="cuda")
    out = cq.kv_attention(q.cuda(), cache, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), lse=lse)
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    for b, n in enumerate(lens):
        at = table[b, :-(-n // page)]
        for i in range(Lq):
            m = n - Lq + i + 1
            if m <= 0:
                assert not out[b, i].any() and np.isneginf(lse[b, i]).all()
                continue
            for h in range(H):
                rows = np.s_[h * G:(h + 1) * G]
                kc, vc = (c[at][:, h].reshape(-1, D)[:m].astype(np.float64) for c in codes)
                ka, va = (s[at][:, h].reshape(-1)[:m] for s in scales)
                case = dict(q=q[b, i, rows].double().numpy(), kf=cols[0][h], vf=cols[1][h], kc=kc, ka=ka, vc=vc, va=va, scale=D ** -0.5, bits=bits)
                worst = sh.worst(out[b, i, rows], lse[b, i, rows], case)
                assert max(worst) <= 1, (b, i, h, worst)
