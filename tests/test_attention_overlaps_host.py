"""Which operands of a call may lie between one another: outputs that share a byte with what is read are refused, and those that only lie next to it, token by token or head
by head, are taken.  Taken calls are refused for a later reason here (no positions), so that no device is needed."""
import random

import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_attention_host import INV, MB, SHAPE, append, cache, desc, refused, rows

BASE = 1 << 30


def takes(status_of_overlap, d, **kw):
    """Whether cf_kv_append takes these operands."""
    with pytest.raises(cf.CFError) as e:
        cf.cf_kv_append(d, cache(), append(n_positions=0, rotary_dim=64, **kw))
    assert e.value.status in (status_of_overlap, SHAPE)
    return e.value.status == SHAPE


@pytest.mark.parametrize("tokens,heads,dim", [(1, 3, 64), (5, 1, 128), (7, 4, 64), (30, 2, 256)])
def test_queries_in_place_between_keys_and_values(tokens, heads, dim):
    d = desc(q_heads=heads, kv_heads=heads, head_dim=dim)
    layouts = {"[tokens, heads, 3, dim]": (heads * 3 * dim, 3 * dim, dim), "[heads, tokens, 3, dim]": (3 * dim, tokens * 3 * dim, dim),
               "[tokens, 3, heads, dim]": (3 * heads * dim, dim, heads * dim), "[heads, 3, tokens, dim]": (dim, 3 * tokens * dim, tokens * dim),
               "[3, tokens, heads, dim]": (heads * dim, dim, tokens * heads * dim), "[3, heads, tokens, dim]": (dim, tokens * dim, tokens * heads * dim)}
    for name, (token, head, part) in layouts.items():
        for order in ((0, 1, 2), (1, 0, 2), (2, 1, 0)):
            q, k, v = (rows(BASE + 2 * i * part, token, head) for i in order)
            assert takes(INV, d, n_tokens=tokens, q=q, q_out=q, k=k, v=v), (name, order)
        # half of a head over its neighbour
        q, k, v = (rows(BASE + 2 * i * part, token, head) for i in range(3))
        for off in (-dim // 2, dim // 2):
            moved = rows(BASE + 2 * part + 2 * off, token, head)
            assert not takes(INV, d, n_tokens=tokens, q=moved, q_out=moved, k=k, v=v) or not overlap(tokens, heads, dim, moved, k) and not overlap(tokens, heads, dim, moved, v), (name, off)


def cells(tokens, heads, x):
    token = 0 if tokens == 1 else x.token
    return [x.data + 2 * (t * token + h * x.head) for t in range(tokens) for h in range(heads)]


def overlap(tokens, heads, dim, x, y):
    ys = sorted(cells(tokens, heads, y))
    import bisect
    for a in cells(tokens, heads, x):
        i = bisect.bisect_left(ys, a - 2 * dim + 1)
        if i < len(ys) and ys[i] < a + 2 * dim:
            return True
    return False


def test_operands_that_share_a_byte_are_never_taken():
    r = random.Random(5)
    taken = apart = 0
    for _ in range(4000):
        tokens, heads, dim = r.randint(1, 6), r.randint(1, 5), 64
        d = desc(q_heads=heads, kv_heads=heads, head_dim=dim)
        unit = r.choice([8, 32, 64, 64])

        def strides():
            parts = r.choice([1, 1, 2, 3, 4])
            forms = [(heads * parts * dim, parts * dim), (parts * dim, tokens * parts * dim), (parts * heads * dim, dim), (dim, parts * tokens * dim),
                     (unit * r.randint(1, 40), unit * r.randint(1, 40))]
            return r.choice(forms)

        token, head = strides()
        other = (token, head) if r.random() < 0.7 else strides()
        q, k = rows(BASE, token, head), rows(BASE + 2 * unit * r.randint(-60, 60), *other)
        inner, outer = sorted(((head, heads), (token, tokens)))
        if inner[0] < dim or outer[0] < (inner[1] - 1) * inner[0] + dim:
            continue                    # not an output's rows: refused for that
        it = takes(INV, d, n_tokens=tokens, q=q, q_out=q, k=k, v=rows(2 * MB, 512, 128))
        meets = overlap(tokens, heads, dim, q, k)
        assert not (it and meets), (tokens, heads, token, head, other, k.data - q.data)
        taken += it
        apart += not meets
    assert taken > 500 and taken > 0.7 * apart
