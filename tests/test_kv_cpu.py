"""The serving operators without a GPU: spans of tables with common beginnings, layouts, and refusals."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

import paper_2609_33224_gb300 as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv():
    P.build()
    from paper_2609_33224_gb300 import kvcache
    return kvcache


def _tree(rng, n):
    """Block tables that branch from common beginnings, unique blocks at their ends."""
    tables, fresh = [], iter(range(1, 1 << 20))
    for _ in range(n):
        t = list(rng.choice(tables))[:rng.randrange(0, 30)] if tables and rng.random() < 0.8 else []
        t += [next(fresh) for _ in range(rng.randrange(1, 20))]
        tables.append(t)
    lengths = [rng.randrange(16 * (len(t) - 1) + 1, 16 * len(t) + 1) for t in tables]
    new = [rng.choice([1, 1, rng.randrange(1, n + 1)]) for n in lengths]
    return tables, lengths, new


@pytest.mark.parametrize("min_blocks", [1, 2, 4])
def test_spans_give_every_query_its_tokens(kv, min_blocks):
    rng = random.Random(min_blocks)
    shared = 0
    for n in (0, 1, 2, 5, 12, 40):
        for _ in range(10):
            tables, lengths, new = _tree(rng, n)
            order, spans, blocks = kv.shared_spans(tables, lengths, new, min_blocks)
            assert sorted(order) == list(range(n))
            q = 0
            for i in order:
                # the request's spans, outermost first, are its table cut in pieces, the last one causal
                mine = sorted((s for s in spans if s["first_query"] <= q < s["first_query"] + s["num_queries"]),
                              key=lambda s: -int(s["num_queries"]) * 2 + int(s["causal"]))
                ids, tokens = [], 0
                for s in mine:
                    nb = -(-int(s["length"]) // 16)
                    ids += list(blocks[int(s["first_block"]):int(s["first_block"]) + nb])
                    tokens += int(s["length"])
                    assert s["first_query"] <= q and q + new[i] <= s["first_query"] + s["num_queries"]
                    assert s["causal"] or s["length"] % 16 == 0
                assert tokens == lengths[i] and ids == tables[i][:-(-lengths[i] // 16)]
                assert [int(s["causal"]) for s in mine] == [0] * (len(mine) - 1) + [1]
                assert mine[-1]["num_queries"] == new[i]
                q += new[i]
            shared += sum(1 for s in spans if not s["causal"])
            assert all(s["causal"] or s["length"] >= 16 * min_blocks for s in spans)
    assert shared > 50


def test_span_refusals(kv):
    for bad in (([[1]], [17], [1]), ([[1]], [3], [0]), ([[1]], [3], [4]), ([[1], [2]], [1], [1])):
        with pytest.raises(ValueError):
            kv.shared_spans(*bad)


def test_struct_layouts_match_c(kv, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text("""
#include <stdio.h>
#include <stddef.h>
#include "packserve_kv.h"
#define P(T) printf(#T " %zu\\n", sizeof(T));
#define O(T, f) printf(#T "." #f " %zu\\n", offsetof(T, f));
int main(void) {
  P(ps_kv_config) P(ps_kv_rows) P(ps_kv_span)
  O(ps_kv_config, num_blocks) O(ps_kv_config, format) O(ps_kv_rows, head_stride) O(ps_kv_rows, type)
  O(ps_kv_span, length) O(ps_kv_span, causal) O(ps_kv_span, first_block)
  return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(line.rsplit(" ", 1) for line in subprocess.run([str(exe)], capture_output=True, text=True,
                                                              check=True).stdout.split("\n") if line)
    ct = {"ps_kv_config": P.PsKvConfig, "ps_kv_rows": P.PsKvRows}
    for k, v in got.items():
        t, _, f = k.partition(".")
        if t == "ps_kv_span":
            assert (kv.SPAN_DTYPE.fields[f][1] if f else kv.SPAN_DTYPE.itemsize) == int(v), k
        else:
            assert (getattr(ct[t], f).offset if f else ctypes.sizeof(ct[t])) == int(v), k


def test_create_without_gpu_reports_an_error(kv):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(P.PSError):
        kv.KVCache(4, 2, 128, device=0)
    L = P.lib()
    out = ctypes.c_void_p()
    assert L.ps_kv_create(None, ctypes.byref(out)) == 1
    for cfg in (P.PsKvConfig(0, 0, 4, 128, 0), P.PsKvConfig(0, 2, 0, 128, 0), P.PsKvConfig(0, 2, 4, 96, 0),
                P.PsKvConfig(0, 2, 4, 128, 3), P.PsKvConfig(0, 2, 4, 128, -1)):
        assert L.ps_kv_create(ctypes.byref(cfg), ctypes.byref(out)) == 1 and not out.value
    # NULL objects are refused, not followed
    assert L.ps_kv_write(None, None, None, None, 0, None) == 1
    assert L.ps_kv_attend(None, None, None, None, None, 1.0, None, 0, None) == 1
    assert L.ps_kv_plan_set(None, 0, None, 0, None, 0) == 1
    L.ps_kv_destroy(None)
    L.ps_kv_plan_destroy(None)
