"""The waits around accesses to a peer CTA's shared memory, by whatever helper they are made: a
kernel that calls a function which maps an address into a peer, or stores, loads or arrives
in the cluster's window, does so behind a cluster barrier, since a peer that has not started has
no memory to write, and the kernels of the orthogonalised updates and 8-bit products pass
one behind their last access, since a peer that has ended has none either."""
import re

import pytest

from tests.test_kernel_waits import REMOTE, _calls, _clean, _functions, _read, _sources

NEWER = ("gemm_i8.cu", "orth_product.cu", "orth_small.cu")
FIRST = {"orth_small.cu": "    cluster_sync();                              // every CTA runs\n",
         "orth_product.cu": "  if (CL > 1 || kSplit) cluster_sync();   // the peers run, and their barriers are initialised before anything arrives on them\n  else",
         "gemm_i8.cu": "  if (CL > 1 || kSplit) cluster_sync();   // the peers run, and their barriers are initialised\n  else"}
LAST = {"orth_product.cu": "  if (CL > 1 || kSplit) cluster_sync();   // the pair's products and arrivals are done in both CTAs; every part's sums are there\n  else",
        "gemm_i8.cu": "  if (CL > 1 || kSplit) cluster_sync();   // the pair's products and arrivals are done in both CTAs; every part's sums are there\n  else"}
# (copies by TMA name the window for their own CTA's memory too)
WINDOW = re.compile(r'"[^"]*\b(?:mapa|st|ld|red|atom|mbarrier\.arrive)\b[\w.]*\.shared::cluster')


def _kernels(text):
    """name -> (positions of accesses to peers, positions of cluster barriers) of a source's kernels."""
    fns = _functions(_clean(text))
    remote = set(REMOTE)
    while True:
        more = {n for n, (k, b) in fns.items() if not k and n not in remote and (_calls(b, remote | {"cluster_addr"}) or WINDOW.search(b))}
        if not more:
            break
        remote |= more
    return {n: (_calls(b, remote), _calls(b, ("cluster_sync", "cluster_wait"))) for n, (k, b) in fns.items() if k}


def unstarted(text):
    return [n for n, (touch, wait) in _kernels(text).items() if touch and (not wait or wait[0] > touch[0])]


def ended(text):
    return [n for n, (touch, wait) in _kernels(text).items() if touch and (not wait or wait[-1] < touch[-1])]


@pytest.mark.parametrize("f", _sources())
def test_peers_have_started(f):
    assert unstarted(_read(f)) == []


@pytest.mark.parametrize("f", NEWER)
def test_peers_have_not_ended(f):
    assert any(touch for touch, _ in _kernels(_read(f)).values()) and ended(_read(f)) == []


@pytest.mark.parametrize("f", NEWER)
def test_a_barrier_taken_out_is_caught(f):
    text = _read(f)
    assert text.count(FIRST[f]) == 1 and text.count(LAST.get(f, FIRST[f])) == 1
    assert unstarted(text.replace(FIRST[f], "  ")) != []
    if f in LAST:   # (the one-launch kernel's accesses all lie between two barriers of a step)
        assert ended(text.replace(LAST[f], "  ")) != []


def test_every_kind_of_access_is_seen():
    kernel = "%s__global__ void __launch_bounds__(32) k(int* p) {\n %s cluster_sync();\n}\n"
    own = '__device__ __forceinline__ void put(int* p) {\n asm volatile("mapa.shared::cluster.u32 %0, %1, %2;");\n}\n'
    there = '__device__ __forceinline__ void put_at(uint32_t at, int v) {\n asm volatile("st.shared::cluster.v4.f32 [%0], %1;");\n}\n'
    through = own + "__device__ __forceinline__ void put_all(int* p) {\n put(p);\n}\n"
    for helper, call in ((there, "put_at(cluster_addr(p, 1), v);"), (own, "put(p);"), (through, "put_all(p);"), ("", "ld_dsmem_f32(p, 1);")):
        assert unstarted(kernel % (helper, call)) == ["k"]
        assert unstarted(kernel % (helper, "cluster_sync(); " + call)) == []
        assert ended(kernel % (helper, "cluster_sync(); " + call)) == []
        assert ended(kernel.replace(" cluster_sync();\n}", "}") % (helper, "cluster_sync(); " + call)) == ["k"]
