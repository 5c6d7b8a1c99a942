"""The serving loop over 8 bits and behind shared instructions: plan, quantising writes and shared attention together, step by step."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300.serving_loop import run  # noqa: E402
from tests.kv8_support import quantise, two  # noqa: E402
from tests.kv_support import UNIT  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("bits,system", [(8, 0), (16, 77), (8, 300)])
def test_attention_sees_the_instructions_and_the_tokens_of_its_request(bits, system):
    """The watcher keeps keys and values itself, as the cache holds them.  A row's bound: the unit roundoff of its result, of its
    weights, and 2^-12 for the FP32 scores (at most 128 products of about 1 and a softmax)."""
    kept, first, seen = {}, {}, [0, 0, 0]
    H, KH, D, u = 8, 2, 64, UNIT[torch.bfloat16]

    def held(x):
        if bits == 16:
            return x.double()
        c, e = quantise(x)
        return c * two(e)[..., None]

    def watch(step, layer, s):
        if step < 0:
            first[layer] = held(s["k"]), held(s["v"])
            return
        got, off = s["kv_len"].cpu().numpy(), np.concatenate([[0], np.cumsum(np.maximum(s["new"], 0))])
        for b, n in enumerate(s["new"]):
            rows = slice(int(off[b]), int(off[b + 1]))
            if n <= 0:
                if n < 0:
                    kept.pop((b, layer), None)
                continue
            out = s["out"][rows].double()
            if got[b] == 0:  # refused: rows without keys, instructions or not
                assert (out == 0).all()
                seen[0] += 1
                continue
            new = held(s["k"][rows]), held(s["v"][rows])
            k, v = (torch.cat([x, y]) for x, y in zip(kept.get((b, layer)) or (y[:0] for y in new), new))
            kept[b, layer] = k, v
            if n > 1 or (b + step) % 4 == 0:
                seen[1 if n > 1 else 2] += 1
                if system:
                    k, v = torch.cat([first[layer][0], k]), torch.cat([first[layer][1], v])
                q = s["q"][rows].double().view(n, KH, H // KH, D)
                x = torch.einsum("tkgd,jkd->kgtj", q, k) / D ** 0.5
                p = torch.arange(len(k) - n, len(k), device="cuda")
                x = x.masked_fill(torch.arange(len(k), device="cuda")[None] > p[:, None], float("-inf"))
                w = torch.softmax(x, -1)
                ref, size = (torch.einsum("kgtj,jkd->tkgd", w, y).reshape(n, H, D) for y in (v, v.abs()))
                assert ((out - ref).abs() <= u * ref.abs() + (u + 2.0 ** -12) * size).all(), (step, layer, b)

    stats = run(steps=50, slots=12, pages=150, layers=2, heads=H, kv_heads=KH, head_dim=D, prompts=(5, 40, 130), watch=watch, bits=bits,
                system=system)
    assert all(seen) and stats["finished"] > 0 and stats["free_pages"] + stats["held_pages"] == stats["pages"]
