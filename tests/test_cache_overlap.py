"""Rotations refuse outputs that share memory with what they read, and pools whose rows share memory (no GPU needed)."""
import ctypes
import subprocess
import textwrap

import pytest

from paper_2609_36938_b200 import binding as B
from paper_2609_36938_b200 import build

INVALID = 1


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


def test_memory_that_is_shared(tmp_path):
    """The rule against a count of every byte."""
    src = tmp_path / "overlap.cpp"
    src.write_text(textwrap.dedent("""
        #include <cstdlib>
        #include <set>
        #include "memory_overlap.h"
        using namespace janus;
        static bool bytes_of(const MoTensor& t, std::set<int64_t>& s) {      // false: some byte twice
            bool once = true;
            for (int64_t i = 0; i < t.n[0]; ++i)
                for (int64_t j = 0; j < t.n[1]; ++j)
                    for (int64_t k = 0; k < t.n[2]; ++k)
                        for (int64_t x = 0; x < t.bytes; ++x) once &= s.insert(t.at + i * t.stride[0] + j * t.stride[1] + k * t.stride[2] + x).second;
            return once;
        }
        int main() {
            std::srand(3);
            int apart = 0, shared = 0;
            for (int n = 0; n < 300000; ++n) {
                MoTensor t[2];
                const int strides[] = {0, 1, 2, 3, 4, 5, 6, 8, 12, 16, 24, 40, 48, 96};
                for (int i = 0; i < 3; ++i) {
                    const int64_t s = strides[std::rand() % 14];
                    for (auto& x : t) {
                        x.n[i] = 1 + std::rand() % 4;
                        x.stride[i] = std::rand() % 4 ? s : strides[std::rand() % 14];
                    }
                }
                for (auto& x : t) {
                    x.at = 1000 + std::rand() % 60;
                    x.bytes = 1 + std::rand() % 8;
                }
                std::set<int64_t> a, b;
                const bool once = bytes_of(t[0], a);
                bytes_of(t[1], b);
                bool same = false;
                for (int64_t x : a) same |= b.count(x) != 0;
                const bool may = mo_may_share(t[0], t[1]);
                if (same != may) return 1;
                if (may != mo_may_share(t[1], t[0])) return 2;
                if (!may) ++apart;
                if (same) ++shared;
                if (mo_apart(t[0]) && !once) return 3;
            }
            return apart > 1000 && shared > 1000 ? 0 : 5;
        }
    """))
    exe = tmp_path / "overlap"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", build.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0


def at(x):
    return ctypes.c_void_p(x)


BASE = 0x10000000      # never dereferenced: validation fails first


def test_rope_refuses_an_output_over_its_input(lib):
    def call(x=BASE, xr=1024, xh=128, T=4, H=8, D=128, out=BASE, outr=1024, outh=128, dt=0):
        return lib.janus_rope(at(x), xr, xh, T, H, D, at(0x1000), at(0x1000), 0, 64, 0, 1.0, 0, dt, at(out), outr, outh, None)

    for bad in (dict(out=BASE + 16), dict(out=BASE - 16), dict(out=BASE + 2048), dict(out=BASE + 2 * 4096 - 2), dict(out=BASE - 2 * 4096 + 2), dict(out=BASE + 256),
                dict(out=BASE + 256, xr=2048, outr=2048), dict(out=BASE + 2 * 1024 - 2, xr=2048, outr=2048), dict(out=BASE + 16, T=1), dict(out=BASE + 16, xr=0, xh=0),
                dict(out=BASE + 16, T=1, H=1), dict(out=BASE + 4, dt=2), dict(out=BASE + 4 * 4096 - 4, dt=2)):
        assert call(**bad) == INVALID, bad


def test_rope_append_refuses_outputs_over_inputs(lib):
    def call(**kw):
        a = dict(q=BASE, qr=1024, qh=128, H=8, k=BASE + 0x100000, kr=512, kh=128, n=4, v=BASE + 0x200000, vr=512, vh=128, T=4, qo=BASE, qor=1024, qoh=128, kp=BASE + 0x400000,
                 kps=32768, kts=512, khs=128, vp=BASE + 0x800000, vps=32768, vts=512, vhs=128, page=64, phys=16)
        a.update(kw)
        return lib.janus_rope_append(at(a["q"]), a["qr"], a["qh"], a["H"], at(a["k"]), a["kr"], a["kh"], a["n"], 128, at(a["v"]), a["vr"], a["vh"], 128, a["T"], at(0x1000),
                                     at(0x1000), at(0x1000), 0, 64, 0, 1.0, at(a["qo"]), a["qor"], a["qoh"], at(a["kp"]), a["kps"], a["kts"], a["khs"], at(a["vp"]), a["vps"],
                                     a["vts"], a["vhs"], a["page"], a["phys"], None, None)

    k, v, kp, vp = BASE + 0x100000, BASE + 0x200000, BASE + 0x400000, BASE + 0x800000
    for bad in (dict(qo=BASE + 16), dict(qo=BASE + 2048), dict(qo=k), dict(qo=k + 512 * 2 * 4 - 16), dict(qo=k - 1024 * 2 * 4 + 16), dict(qo=v), dict(qo=v + 256), dict(qo=kp + 512), dict(qo=vp + 1024),
                # rows of a fused projection: the queries' places reach into the keys'
                dict(q=BASE, qr=2048, qo=BASE + 16 * 7 * 16, qor=2048, k=BASE + 2 * 1024, kr=2048, v=BASE + 2 * 1536, vr=2048),
                # values into rows of the keys
                dict(vp=kp + 16), dict(vp=kp + 32768 * 2 * 15), dict(vp=kp + 128, kts=1024, vts=1024, kps=65536, vps=65536),
                # pages that share rows
                dict(kps=0), dict(kps=512), dict(vps=32760), dict(kps=64), dict(vps=0)):
        assert call(**bad) == INVALID, bad


def test_large_tensors_are_decided(tmp_path):
    """Layouts of real sizes: pages that hold keys and then values of another width, interleaved rows, slices of a projection, heads outermost; and each a byte further on."""
    src = tmp_path / "layouts.cpp"
    src.write_text(textwrap.dedent("""
        #include "memory_overlap.h"
        using namespace janus;
        int main() {
            const int64_t pages = 100000, page = 64, n = 16, dk = 384, dv = 256, T = 8192;
            const uintptr_t at = uintptr_t(1) << 40;
            const int64_t block = page * n * (dk + dv);
            // keys of a page, then its values
            MoTensor k = {at, dk, {pages, page, n}, {block, n * dk, dk}}, v = {at + page * n * dk, dv, {pages, page, n}, {block, n * dv, dv}};
            if (mo_may_share(k, v)) return 1;
            v.at -= 1;
            if (!mo_may_share(k, v)) return 2;
            v.at += 2;      // the last value reaches into the next page's first key
            if (!mo_may_share(k, v)) return 3;
            // keys and values of a head beside each other, heads outermost
            k = {at, dk, {pages, page, n}, {page * (dk + dv), dk + dv, pages * page * (dk + dv)}};
            v = {at + dk, dv, {pages, page, n}, {page * (dk + dv), dk + dv, pages * page * (dk + dv)}};
            if (mo_may_share(k, v)) return 4;
            v.at -= 1;
            if (!mo_may_share(k, v)) return 5;
            // queries, keys and values of a projection; a row of values as they follow one another
            const MoTensor q = {at, 256, {T, 32, 1}, {48 * 256, 256, 0}};
            MoTensor kk = {at + 32 * 256, 256, {T, 8, 1}, {48 * 256, 256, 0}};
            if (mo_may_share(q, kk)) return 6;
            kk.at -= 16;
            if (!mo_may_share(q, kk)) return 7;
            // layers of one pool, far apart and interleaved
            const MoTensor a = {at, 1152, {pages, page, 1}, {int64_t(61) * page * 1152, 1152, 0}};
            MoTensor b = {at + page * 1152, 1152, {pages, page, 1}, {int64_t(61) * page * 1152, 1152, 0}};
            if (mo_may_share(a, b)) return 8;
            b.at -= 2;
            if (!mo_may_share(a, b)) return 9;
            return 0;
        }
    """))
    exe = tmp_path / "layouts"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", build.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0
