"""The serving loop: every page is accounted for, and each step's attention is that of the tokens each request wrote."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300.serving_loop import run  # noqa: E402
from tests.kv_support import UNIT  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def test_attention_sees_the_tokens_of_its_request():
    """The watcher keeps each request's keys and values itself.  A row's bound: the unit roundoff of its result, of its
    weights, and 2^-12 for the FP32 scores (at most 128 products of about 1 and a softmax)."""
    kept, seen = {}, [0, 0, 0]
    H, KH, D = 8, 2, 64

    def watch(step, layer, s):
        got, off = s["kv_len"].cpu().numpy(), np.concatenate([[0], np.cumsum(np.maximum(s["new"], 0))])
        for b, n in enumerate(s["new"]):
            rows = slice(int(off[b]), int(off[b + 1]))
            if n <= 0:
                if n < 0:
                    kept.pop((b, layer), None)
                continue
            out = s["out"][rows].double()
            if got[b] == 0:  # refused: rows without keys
                assert (out == 0).all() and (s["pos"][rows] == -1).all()
                seen[0] += 1
                continue
            k0, v0 = kept.get((b, layer), (s["k"][:0], s["v"][:0]))
            k, v = torch.cat([k0, s["k"][rows]]), torch.cat([v0, s["v"][rows]])
            kept[b, layer] = k, v
            assert len(k) == got[b] and s["pos"][rows].tolist() == list(range(got[b] - n, got[b]))
            if b % 3 == step % 3:
                seen[1 if n > 1 else 2] += 1
                q = s["q"][rows].double().view(n, KH, H // KH, D)
                x = torch.einsum("tkgd,jkd->kgtj", q, k.double()) / D ** 0.5
                p = torch.arange(got[b] - n, got[b], device="cuda")
                x = x.masked_fill(torch.arange(got[b], device="cuda")[None] > p[:, None], float("-inf"))
                w = torch.softmax(x, -1)
                ref = torch.einsum("kgtj,jkd->tkgd", w, v.double()).reshape(n, H, D)
                tol = UNIT[torch.bfloat16] * ref.abs() + (UNIT[torch.bfloat16] + 2.0 ** -12) * \
                    torch.einsum("kgtj,jkd->tkgd", w, v.double().abs()).reshape(n, H, D)
                assert ((out - ref).abs() <= tol).all(), (step, layer, b)

    stats = run(steps=60, slots=12, pages=150, layers=2, heads=H, kv_heads=KH, head_dim=D, prompts=(5, 40, 130), watch=watch)
    assert all(seen) and stats["refused_new"] > 0 and stats["finished"] > 0
    assert stats["free_pages"] + stats["held_pages"] == stats["pages"]
    assert stats["tokens"] > stats["admitted"] > 0
