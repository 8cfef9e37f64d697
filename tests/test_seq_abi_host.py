"""Host-side checks of the sequence operators' C ABI (no GPU needed): every
entry point that include/snn_seq.h declares is exported, the ctypes mirror has
its layouts, and what create refuses is refused before the device is touched."""
import ctypes as C
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    import paper_2501_07331_amd as snn
    from paper_2501_07331_amd import sequence
    return sequence._bind(snn.load_library())


def _header():
    return open(os.path.join(ROOT, "include", "snn_seq.h")).read()


def test_every_declared_symbol_is_exported(lib):
    names = set(re.findall(r"\b(snn_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", _header(), flags=re.S)))
    assert {"snn_seq_create", "snn_seq_scan_backward", "snn_sampler_sample"} <= names
    for n in names:
        assert hasattr(lib, n), n


def test_struct_layouts_and_constants_match_header(tmp_path):
    from paper_2501_07331_amd import sequence as b
    structs = [b.snn_tensor, b.snn_seq_opts, b.snn_seq_conv, b.snn_seq_conv_grad, b.snn_seq_scan, b.snn_seq_scan_grad,
               b.snn_sample_args]
    consts = [n for n in dir(b) if re.match(r"SNN_(SEQ|SAMPLE|F32|BF16|F16|E4M3)", n)]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "snn_seq.h"', 'int main(void) {']
    for st in structs:
        lines.append(f'  printf("{st.__name__} %zu\\n", sizeof({st.__name__}));')
        lines += [f'  printf("{st.__name__}.{f} %zu\\n", offsetof({st.__name__}, {f}));' for f, _ in st._fields_]
    lines += [f'  printf("{n} %zu\\n", (size_t){n});' for n in consts] + ['  return 0;', '}']
    (tmp_path / "probe.c").write_text("\n".join(lines) + "\n")
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(tmp_path / "probe.c")], check=True)
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for st in structs:
        assert int(got[st.__name__]) == C.sizeof(st), st.__name__
        for f, _ in st._fields_:
            assert int(got[f"{st.__name__}.{f}"]) == getattr(st, f).offset, (st.__name__, f)
    for n in consts:
        assert int(got[n]) == getattr(b, n), n


@pytest.mark.parametrize("kw", [dict(batch=0), dict(batch=65536), dict(T=0), dict(T=65537), dict(channels=0),
                                dict(channels=65537), dict(state=0), dict(state=65), dict(groups=0), dict(groups=4),
                                dict(taps=0), dict(taps=9), dict(flags=4), dict(flags=2), dict(batch=40000, T=65536)])
def test_create_refuses(lib, kw):
    from paper_2501_07331_amd import sequence as b
    o = b.snn_seq_opts(**dict(dict(batch=2, T=10, channels=6, state=4, groups=2, taps=4, flags=0, hip_stream=None), **kw))
    h = C.c_void_p(123)
    assert lib.snn_seq_create(C.byref(o), C.byref(h)) == -1
    assert h.value is None and lib.snn_seq_last_error(None)


def test_null_handles_are_refused(lib):
    assert lib.snn_seq_create(None, None) == -1
    for f in (lib.snn_seq_conv_forward, lib.snn_seq_conv_backward, lib.snn_seq_conv_step, lib.snn_seq_scan_forward,
              lib.snn_seq_scan_backward, lib.snn_seq_scan_step, lib.snn_sampler_sample, lib.snn_seq_saved):
        assert f(None, None) == -1
    assert lib.snn_seq_pack(None, 1, None, None) == -1 and lib.snn_seq_unpack(None, 1, None, None) == -1
    assert lib.snn_seq_bin_spikes(None, None, 1, 1, None) == -1
    assert lib.snn_seq_bin_records(None, None, 1, 1, 1, None) == -1
    lib.snn_seq_destroy(None)
    lib.snn_sampler_destroy(None)


@pytest.mark.parametrize("rows,n", [(0, 5), (-1, 5), (3, 0), (3, (1 << 24) + 1)])
def test_sampler_create_refuses(lib, rows, n):
    h = C.c_void_p(123)
    assert lib.snn_sampler_create(rows, n, None, C.byref(h)) == -1
    assert h.value is None and lib.snn_sampler_last_error(None)
