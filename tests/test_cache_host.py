"""The paged cache's host side: the header and the binding agree, every refusal comes before any device work, and pages
have the owners that a plain model of them says.  No GPU."""
import ctypes
import os
import random
import re

import numpy as np
import pytest

from paper_2406_11209_amd import api, cache
from paper_2406_11209_amd.api import Codec, PbzError

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20          # an address that is aligned and never read: every call below is refused before a launch


def test_the_binding_covers_the_header():
    text = open(os.path.join(ROOT, "include", "pbz_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(pbz_[a-z0-9_]+)\s*\(", text)))
    assert sorted(cache.SIGNATURES) == names
    lib = cache._library()
    for name in names:
        assert hasattr(lib, name), name
    for code in (-14, -15, -16, -17):
        assert api.status_string(code) != "unknown status"


def geometry(**changes):
    fields = dict(n_pages=8, heads=2, page_size=16, k_N=FAKE, k_F=FAKE, v_N=FAKE, v_F=FAKE)
    fields.update(changes)
    return cache._Cache(**fields)


@pytest.mark.parametrize("codec, status", [
    (lambda: Codec((128,)), 0), (lambda: Codec((32,), "f16"), 0), (lambda: Codec((256,), "bf16", transform="haar"), 0),
    (lambda: Codec((16,)), -3), (lambda: Codec((1, 128)), -3), (lambda: Codec((128,), "f64"), -4),
    (lambda: Codec((128,), "f32", "i16"), -4), (lambda: Codec((32,), mask=np.arange(32) < 31), -17)])
def test_codecs_that_a_cache_takes(codec, status):
    c = codec()
    assert cache._library().pbz_cache_layout(c._h, geometry(), None, None) == status


def test_layout():
    n, f = ctypes.c_size_t(), ctypes.c_size_t()
    lib = cache._library()
    assert lib.pbz_cache_layout(Codec((64,), "f16")._h, geometry(), n, f) == 0
    assert (n.value, f.value) == (8 * 2 * 16 * 2, 8 * 2 * 16 * 64)
    assert lib.pbz_cache_layout(None, geometry(), n, f) == -1
    assert lib.pbz_cache_layout(Codec((64,))._h, None, n, f) == -1
    for bad in (dict(n_pages=0), dict(n_pages=1 << 31), dict(heads=0), dict(heads=65536), dict(page_size=8), dict(page_size=48),
                dict(page_size=2048), dict(page_size=0), dict(n_pages=1 << 30, heads=1024, page_size=1024)):
        assert lib.pbz_cache_layout(Codec((64,))._h, geometry(**bad), n, f) == -7, bad


def test_append_refusals():
    c, lib = Codec((64,)), cache._library()
    x = cache._Lines(FAKE, 128, 64)

    def call(codec=c, g=geometry(), tokens=3, k=x, v=x, dtype=api.PBZ_BF16, slots=FAKE):
        return lib.pbz_cache_append(codec._h if codec else None, g, tokens, k, v, dtype, slots, None)

    assert call(codec=None) == -1 and call(g=None) == -1 and call(k=None) == -1 and call(slots=None) == -1
    assert call(v=cache._Lines(None, 128, 64)) == -1
    for name in ("k_N", "k_F", "v_N", "v_F"):
        assert call(g=geometry(**{name: None})) == -1
        assert call(g=geometry(**{name: FAKE + 8})) == -14
    assert call(dtype=4) == -4 and call(dtype=-1) == -4
    assert call(tokens=0) == -7 and call(tokens=-1) == -7 and call(tokens=1 << 31) == -7
    assert call(k=cache._Lines(FAKE, -1, 64)) == -7 and call(v=cache._Lines(FAKE, 128, -64)) == -7
    assert call(k=cache._Lines(FAKE, 1 << 41, 64)) == -7


def test_copy_refusals():
    c, lib = Codec((64,)), cache._library()

    def call(pairs, n=None, g=geometry(n_pages=100)):
        a = np.asarray(pairs, dtype=np.int32).reshape(-1, 2)
        return lib.pbz_cache_copy_pages(c._h, g, len(a) if n is None else n, a.ctypes.data, None)

    assert lib.pbz_cache_copy_pages(c._h, geometry(), 1, None, None) == -1
    assert call([(0, 1)], n=0) == -7 and call([(0, 1)], n=101) == -7
    for pairs in ([(0, 100)], [(-1, 3)], [(100, 3)], [(3, 3)], [(1, 2), (4, 2)], [(1, 2), (2, 5)], [(2, 5), (1, 2)]):
        assert call(pairs) == -15, pairs
        many = [(i, 50 + i) for i in range(10, 45)]                   # beyond the number up to which pairs are compared one by one
        assert call(many + pairs) == -15, pairs


def attention(**changes):
    fields = dict(q=FAKE, out=FAKE, lengths=FAKE, table=FAKE, starts=FAKE, type=api.PBZ_BF16, q_heads=4, q_token_stride=256,
                  q_head_stride=64, out_token_stride=256, out_head_stride=64, n_tokens=5, n_seqs=2, table_stride=4,
                  max_pages=4, max_new=3, causal=1, scale=0.125)
    fields.update(changes)
    return cache._Attention(**fields)


def test_attend_refusals():
    c, lib = Codec((64,)), cache._library()
    need = ctypes.c_size_t()
    assert lib.pbz_cache_attend_workspace(c._h, geometry(), attention(), need) == 0 and need.value > 0

    def call(a, g=geometry(), ws=FAKE, size=1 << 40):
        return lib.pbz_cache_attend(c._h, g, a, ws, size, None)

    assert lib.pbz_cache_attend(None, geometry(), attention(), FAKE, 1 << 40, None) == -1
    assert lib.pbz_cache_attend_workspace(c._h, geometry(), attention(), None) == -1
    assert call(None) == -1 and call(attention(), ws=None) == -1
    for name in ("q", "out", "lengths", "table"):
        assert call(attention(**{name: None})) == -1, name
    assert call(attention(), g=geometry(v_F=FAKE + 4)) == -14
    assert call(attention(), size=need.value - 1) == -8 and call(attention(), ws=FAKE + 8) == -8
    for dtype in (api.PBZ_F64, api.PBZ_F32, 9):
        assert call(attention(type=dtype)) == -4
    for scale in (float("nan"), float("inf")):
        assert call(attention(scale=scale)) == -9
    for bad in (dict(q_heads=3), dict(q_heads=0), dict(n_tokens=0), dict(n_seqs=0), dict(max_pages=0), dict(table_stride=3),
                dict(max_new=0), dict(max_length=-1), dict(window=-1), dict(window=1 << 31), dict(starts=None),
                dict(max_pages=1 << 27, table_stride=1 << 27), dict(n_tokens=1 << 30), dict(q_token_stride=-1),
                dict(out_head_stride=-1), dict(q_head_stride=1 << 41), dict(n_seqs=1 << 31)):
        assert call(attention(**bad)) == -7, bad


def test_pages_refusals():
    for args in ((0, 16), (-1, 16), (1 << 31, 16), (4, 8), (4, 24), (4, 2048)):
        with pytest.raises(PbzError) as e:
            cache.Pages(*args)
        assert e.value.status == -7
    lib = cache._library()
    assert lib.pbz_pages_create(None, 4, 16) == -1
    lib.pbz_pages_destroy(None)
    p = cache.Pages(4, 16)
    a = p.open()
    for call in (lambda: p.fork(a + 1), lambda: p.close(a + 1), lambda: p.extend(a + 1, 1), lambda: p.truncate(a + 1, 0),
                 lambda: p.length(a + 1), lambda: p.table(a + 1)):
        with pytest.raises(PbzError) as e:
            call()
        assert e.value.status == -16
    for tokens in (0, -1, 1 << 31):
        with pytest.raises(PbzError) as e:
            p.extend(a, tokens)
        assert e.value.status == -7
    p.extend(a, 40)
    with pytest.raises(PbzError) as e:                  # two of four pages more than there are
        p.extend(a, 25)
    assert e.value.status == -15 and p.length(a) == 40 and p.free_count == 1
    for length in (-1, 41):
        with pytest.raises(PbzError) as e:
            p.truncate(a, length)
        assert e.value.status == -7
    with pytest.raises(PbzError) as e:
        p.table(a, 2)
    assert e.value.status == -13
    # a fork in the middle of a page needs a page to write even one token, a fork at its end does not need a copy
    b = p.fork(a)
    p.extend(a, 8)                                       # takes the last page for its own copy
    assert p.free_count == 0
    with pytest.raises(PbzError) as e:
        p.extend(p.fork(a), 1)
    assert e.value.status == -15
    p.close(a)
    assert p.length(b) == 40
    slots, copy = p.extend(b, 8)                         # nobody shares b's last page any more ... but the fork of a holds its own
    assert copy is None and len(slots) == 8


class Model:
    """Pages as a plain dict: what every position of every sequence holds, page by page."""

    def __init__(self, n_pages, size):
        self.size, self.content, self.seqs = size, {}, {}

    def check(self, pages):
        """Every sequence's slots hold what it wrote or inherited."""
        owners = {}
        for seq, tokens in self.seqs.items():
            table = pages.table(seq)
            assert pages.length(seq) == len(tokens) and len(table) == -(-len(tokens) // self.size)
            assert len(set(table.tolist())) == len(table)
            for j, token in enumerate(tokens):
                assert self.content[int(table[j // self.size]) * self.size + j % self.size] == token
            for page in table.tolist():
                owners.setdefault(page, set()).add(seq)
        assert pages.free_count == pages.n_pages - len(owners)

    def copy(self, pairs):
        reads = {int(a): [self.content.get(int(a) * self.size + i) for i in range(self.size)] for a, _ in pairs}
        for a, b in pairs:
            for i in range(self.size):
                self.content[int(b) * self.size + i] = reads[int(a)][i]


@pytest.mark.parametrize("seed", range(6))
def test_pages_against_a_model(seed):
    rng = random.Random(seed)
    size, n_pages = 16, rng.choice([3, 17, 40])
    pages, model, count = cache.Pages(n_pages, size), Model(n_pages, size), 0
    for _ in range(400):
        action = rng.random()
        seqs = list(model.seqs)
        if action < 0.15 or not seqs:
            model.seqs[pages.open()] = []
        elif action < 0.6:
            seq, n = rng.choice(seqs), rng.randrange(1, 50)
            try:
                slots, copy = pages.extend(seq, n)
            except PbzError as e:
                assert e.status == -15
                continue
            if copy:
                model.copy([copy])
            for slot in slots.tolist():
                model.content[slot] = count
                model.seqs[seq].append(count)
                count += 1
        elif action < 0.75:
            seq = rng.choice(seqs)
            model.seqs[pages.fork(seq)] = list(model.seqs[seq])
        elif action < 0.85:
            seq = rng.choice(seqs)
            pages.close(seq)
            del model.seqs[seq]
        elif action < 0.93:
            seq = rng.choice(seqs)
            n = rng.randrange(len(model.seqs[seq]) + 1)
            pages.truncate(seq, n)
            del model.seqs[seq][n:]
        else:
            pairs = pages.compact()
            model.copy(pairs.tolist())
            assert not set(pairs[:, 0].tolist()) & set(pairs[:, 1].tolist())
            used = n_pages - pages.free_count
            assert all(p < used for s in model.seqs for p in pages.table(s).tolist())
        model.check(pages)


def test_compact_says_when_there_is_no_room_for_the_moves():
    p = cache.Pages(8, 16)
    a, b = p.open(), p.open()
    p.extend(a, 48)
    p.extend(b, 48)
    p.close(a)
    pairs, n = np.zeros((8, 2), np.int32), ctypes.c_int64()
    lib = cache._library()
    assert lib.pbz_pages_compact(p._h, pairs.ctypes.data, 2, n) == -13
    assert sorted(p.table(b).tolist()) == [3, 4, 5]
    assert lib.pbz_pages_compact(p._h, pairs.ctypes.data, 3, n) == 0 and n.value == 3
    assert sorted(p.table(b).tolist()) == [0, 1, 2]
