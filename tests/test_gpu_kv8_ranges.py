"""Caches of 8 bits at the ends of their ranges."""

import copy

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import Case8, Shared  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


def spoil_page_zero(case, *tables):
    """Nobody holds page 0 (what it held moves to a page that nobody has), and nobody wrote it: NaN codes, scale bytes of 255."""
    free = set(range(case.codes[0].shape[0])) - set(case.table[case.table >= 0].tolist())
    if 0 not in free:
        to = min(free)
        for a in (*case.codes, *case.exps):
            a[to] = a[0]
        for t in (case.table, *tables):
            t[t == 0] = to
    for a, x in zip((*case.codes, *case.exps), (0x7f, 0x7f, 255, 255)):
        a[0] = x


def without(case, b, first, n):
    """The case as ``check`` takes it, positions first .. first + n - 1 of request b, which all of its rows would see, left out."""
    c = copy.copy(case)
    c.lens, c.keys, c.values = list(case.lens), list(case.keys), list(case.values)
    q, kv = c.lens[b]
    assert kv - q >= first + n
    c.lens[b] = (q, kv - n)
    for x in (c.keys, c.values):
        x[b] = torch.cat([x[b][:first], x[b][first + n:]])
    return c


def reported(ctx):
    with pytest.raises(kvdro.KvdroError) as e:
        kvdro.kvdro_sync(ctx)
    assert e.value.status == kvdro.KVDRO_ERANGE


@pytest.mark.parametrize("q", [1, 3, 6, 20, 300])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 32), ("bf16", 64, 128), ("fp16", 128, 64)])
@pytest.mark.parametrize("opt", [{}, {"softcap": 30.0}], ids=["plain", "cap"])
def test_a_page_that_is_none_is_left_out(ctx, q, dtype, D, page, opt):
    """In the middle of a request, where every row sees the whole block; nothing of any other page takes its place."""
    case = Case8([(q, 1500), (1, 100)], dtype, D, 8, 2, page, seed=q)
    spoil_page_zero(case)
    for bad in (-1, 10 ** 6):
        case.table[0, 2] = bad
        out, lse = case.run(ctx, **opt)
        reported(ctx)
        without(case, 0, 2 * page, page).check(out, lse, **opt)


@pytest.mark.parametrize("lens", [[(1, 100), (1, 30)], [(1, 100)] * 12, [(40, 90), (1, 30)]], ids=["few", "tokens", "chunk"])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 32)])
def test_a_page_of_a_prefix_that_is_none_is_left_out(ctx, lens, wide, dtype, D, page):
    s = Shared(lens, [0, len(lens)], [700], bits=8, wide=wide, dtype=dtype, D=D, Hq=8, Hkv=2, page=page, seed=2)
    spoil_page_zero(s.c, s.table, s.prefix_table)
    s.prefix_table[0, 3] = -1
    out, lse = s.run(ctx)
    reported(ctx)
    for x in (s.c.keys, s.c.values):
        x[s.B] = torch.cat([x[s.B][:3 * page], x[s.B][4 * page:]])
    s.check(out, lse)
