"""The plan of a batch with masked spans: its pieces give every query all of such a span's keys, and both kernels are told where
the own ones begin; the tile kernel takes those of a limited number of queries."""
import os
import random
import subprocess

import pytest

from tests import test_kv_plan_host as host


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "p.cpp", d / "p"
    text = host.HARNESS
    for old, new in (
            # the own tokens are the mask's: a query's pieces reach to the span's end
            ("const long lim = s->causal ?", "const bool masked = s->causal == kMasked;\n"
             "          CHECK(kind || p.split == (masked ? 1u : 0u));\n"
             "          if (masked && !kind) CHECK((long)p.climit == (long)s->length - (long)s->num_queries);\n"
             "          if (kind && p.climit == kNoLimit) CHECK(!masked || last <= (long)s->length - (long)s->num_queries);\n"
             "          else if (kind) CHECK(masked && o.mask_tiles && s->num_queries <= kTileOwn && (long)p.climit == (long)s->length - (long)s->num_queries);\n"
             "          else CHECK(!masked || o.mask_rows);\n"
             "          const long lim = masked ? (long)s->length : s->causal ?"),
            ("else CHECK((long)p.climit ==", "else if (!masked) CHECK((long)p.climit =="),
            (": s.causal ? std::min<long>", ": s.causal == 1 ? std::min<long>"),
            ("x < (p.split ? 2u : 1u)", "x < (kind && p.split ? 2u : 1u)"),
            ("if (p.split) CHECK(kind &&", "if (kind && p.split) CHECK(kind &&"),
            # pieces side by side are neighbours of one worker, of one tile of rows each, and no piece is in two pairs
            ("const unsigned step = kind ? kTileKeys : kBlock;", "const unsigned step = kind ? kTileKeys : kBlock;\n"
             "        if (kind && p.fold0) {\n"
             "          const size_t at = &p - pieces.data(), w = std::upper_bound(off.begin(), off.end(), at) - off.begin();\n"
             "          CHECK(o.mask_tiles && at + 1 < off[w] && !pieces[at + 1].fold0 && p.fold0 == 1);\n"
             "          for (size_t x = at; x < at + 2; ++x) CHECK(!pieces[x].split && (int)pieces[x].nrows <= tile_rows_of(D) / 2);\n"
             "          ++pairs;\n"
             "        }"),
            ("const unsigned workers = kind ?", "unsigned pairs = 0;\n      const unsigned workers = kind ?"),
            ("        if (p.nfold) CHECK(next == p.nrows);\n      }\n", "        if (p.nfold) CHECK(next == p.nrows);\n      }\n"
             "      CHECK(!kind || pairs == o.pairs);\n")):
        assert text.count(old) == 1, old
        text = text.replace(old, new)
    src.write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", host.CSRC, "-I", os.path.join(host.ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)

    def run(cases):
        text = ""
        for (sms, D, fmt, H, g, T), spans in cases:
            text += "%d %d %d %d %d %d %d\n" % (sms, D, fmt, H, g, T, len(spans)) + "".join("%d %d %d %d\n" % s for s in spans)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == len(cases), (cases[len(lines) - 1], lines[-1:])
        return [tuple(int(x) for x in ln.split()[1:]) for ln in lines]
    return run


def _random(rng):
    shape, spans = host._random(rng)
    if rng.random() < 0.2:  # more own tokens than the tile kernel takes
        shape = (*shape[:5], 600)
        spans = [(0, 600, 2000, 2), (10, 257, 257, 2), (300, 256, 900, 2)]
    return shape, [(a, n, max(length, n), 2) if rng.random() < 0.6 else (a, n, length, c) for a, n, length, c in spans]


def test_every_key_once(plan):
    rng = random.Random(5)
    got = plan([_random(rng) for _ in range(400)])
    assert any(x[1] for x in got) and any(x[0] for x in got) and any(x[2] for x in got)


def test_forms(plan):
    got = plan([
        # contexts and drafts by tiles
        ((152, 128, 0, 8, 8, 640), [(64 * i, 64, 4000 + 64 + i, 2) for i in range(10)]),
        # drafts on a shared prefix
        ((152, 128, 2, 8, 8, 310), [(0, 310, 16384, 0)] + [(31 * i, 31, 31 + i, 2) for i in range(10)]),
        # joined in by the row kernel
        ((4, 128, 0, 2, 8, 300), [(0, 300, 500, 0)] + [(i * 30, 30, 60, 2) for i in range(10)]),
        # alone: written by the row kernel
        ((152, 64, 1, 1, 1, 16), [(0, 16, 16, 2)]),
        # many of one tile
        ((152, 128, 0, 8, 8, 512), [(16 * i, 16, 916 + i, 2) for i in range(32)]),
    ])
    assert not got[4][0] and got[4][1]
    assert not got[0][0] and got[0][1] and got[1][0] and got[1][1]
    assert got[2][3] > 0
    assert got[3] == (1, 0, 0, 0)
