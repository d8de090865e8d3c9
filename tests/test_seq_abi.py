"""CPU-side checks of the calls that use the cache: the binding's structures lie as the header's do, and what the binding
refuses it refuses before any GPU work."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structures_lie_as_in_the_header(tmp_path):
    from paper_2609_39358_b200 import binding
    pairs = {"gk_batch": binding.CBatch, "gk_rows": binding.CRows, "gk_rope": binding.CRope}
    lines = []
    for name, cls in pairs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gk.h"\nint main(void) {' + "\n".join(lines) +
                   'printf("%u %u\\n", GK_SEQ_POSITION, GK_ATTN_FULL); return 0; }')
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = subprocess.check_output([str(exe)], text=True).split()
    want = []
    for cls in pairs.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert [int(x) for x in out[:-2]] == want
    assert [int(x) for x in out[-2:]] == [binding.SEQ_POSITION, binding.GK_ATTN_FULL]


def test_null_contexts_are_refused():
    from paper_2609_39358_b200 import build, load_library
    build.build()
    lib = load_library()
    assert lib.gk_append(None, None, 0, None, None, None, None, 0, None, None, None) == -1
    assert lib.gk_attention(None, None, 0, None, 0, None, None, None, 1.0, 0, 0, None) == -1


def test_batches_and_rotations_are_checked():
    import paper_2609_39358_b200 as gk
    table, kv = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    start = torch.zeros(3, dtype=torch.int32)
    assert gk.Batch(table, kv).n_tokens == 2
    b = gk.Batch(table, kv, start, 9)
    assert (b.n_seqs, b.n_tokens, b.max_q_len) == (2, 9, 9)
    for bad in (lambda: gk.Batch(table.long(), kv), lambda: gk.Batch(table[:1], kv), lambda: gk.Batch(table, kv, start),
                lambda: gk.Batch(table, kv, start[:2], 4), lambda: gk.Batch(table, kv, n_tokens=5),
                lambda: gk.Batch(table.t(), torch.zeros(3, dtype=torch.int32)),
                lambda: gk.Batch(table, kv, status=torch.zeros(1, dtype=torch.uint8)),
                lambda: gk.Rope(torch.zeros(4, 32).double()), lambda: gk.Rope(torch.zeros(4, 32), sections=(4, 4, 4, 4)),
                lambda: gk.Rope(torch.zeros(4, 32), sections=(8, 8), positions=torch.zeros(3, 2, dtype=torch.int32))):
        with pytest.raises(gk.GkError) as e:
            bad()
        assert e.value.code == -1


def test_a_cache_is_marshalled_anew_when_it_changes():
    import paper_2609_39358_b200 as gk
    from paper_2609_39358_b200.binding import CCache
    c = gk.Cache(torch.zeros(64, dtype=torch.uint8), 4, 32, 16, 8)
    first = c.ref()
    assert c.ref() == first and CCache.from_address(first).num_pages == 4
    c.num_pages = 7
    assert CCache.from_address(c.ref()).num_pages == 7
    c.data = torch.zeros(128, dtype=torch.uint8)
    assert CCache.from_address(c.ref()).data == c.data.data_ptr()
