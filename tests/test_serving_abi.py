"""CPU checks of the entry points that end a serving step: arguments are refused with a
status and a message before any device is touched; workspace sizes; the binding's own
checks; the oracle's page tables keep what they promise."""
import ctypes
import random

import pytest
import torch

import serving
from paper_2607_27042_amd import binding, build


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return binding.load()


NULL = ctypes.c_void_p(0)
P = ctypes.c_void_p(4096)  # aligned, never followed: every call here is refused
F32, F64, BF16 = binding.F32, binding.F64, binding.BF16


def refused(status, part):
    assert status == -1, status
    assert part in binding.gptq2d_last_error(), binding.gptq2d_last_error()


def test_verify_refusals(lib):
    size = lib.gptq2d_tree_verify_workspace_size
    assert size(2, 65, 100) == 0 and size(0, 3, 100) == 0 and size(2, 3, 0) == 0 and size(2, 3, 100) > 0
    ok = dict(seqs=2, width=3, vocab=100, dt=BF16, X=P, ldx=100, scale=1.0, tokens=P, parents=P, drafts=P, u=P, D=P, ldd=100,
              ds=1.0, dlse=P, path=P, count=P, next=P, lp=P, ws=P, nb=size(2, 3, 100), stream=None)
    call = lambda **k: lib.gptq2d_tree_verify(*{**ok, **k}.values())
    refused(call(seqs=-1), "seqs")
    refused(call(seqs=65536), "seqs")
    refused(call(width=0), "width")
    refused(call(width=65), "width")
    refused(call(vocab=2 ** 28 + 1), "vocab")
    refused(call(dt=F64), "dtype")
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        refused(call(scale=bad), "scale")
        refused(call(ds=bad), "draft_scale")
    refused(call(dlse=NULL), "draft_lse")
    refused(call(u=NULL), "random numbers")
    for name in ("X", "tokens", "path", "count", "next", "lp"):
        refused(call(**{name: NULL}), "NULL")
    refused(call(ldx=99), "leading dimension")
    refused(call(ldd=99), "leading dimension")
    refused(call(X=ctypes.c_void_p(4097)), "aligned")
    refused(call(next=ctypes.c_void_p(4100)), "aligned")
    assert call(seqs=0) == 0  # no work
    assert call(nb=ok["nb"] - 1) == -6 and call(ws=NULL) == -6 and call(ws=ctypes.c_void_p(4100)) == -6


def arrays(n, **null):
    """Host arrays of the layers' tensors; null: name -> the layer whose pointer is other."""
    out = []
    for name in ("KC", "VC", "KS", "VS"):
        a = (ctypes.c_void_p * n)(*[4096] * n)
        if name in null:
            a[null[name][0]] = null[name][1]
        out.append(a)
    return out


def test_commit_and_copy_refusals(lib):
    def commit(layers=3, seqs=2, width=4, heads=2, dim=64, pages=4, page=16, of=None, table=P, ldt=4, tw=4, context=P, path=P):
        return lib.gptq2d_cache_commit(layers, seqs, width, heads, dim, pages, page, *(of or arrays(3)), table, ldt, tw, context,
                                       path, None)

    def copy(layers=3, count=2, heads=2, dim=64, pages=4, page=16, of=None, copies=P):
        return lib.gptq2d_cache_copy(layers, count, heads, dim, pages, page, *(of or arrays(3)), copies, None)

    for call in (commit, copy):
        refused(call(layers=0), "layers")
        refused(call(layers=4097), "layers")
        refused(call(heads=0), "heads")
        refused(call(dim=24), "dim")
        refused(call(page=8), "page_size")
        refused(call(pages=2 ** 31 // 16), "tokens")
        refused(call(of=[None] + arrays(3)[1:]), "NULL")
        refused(call(of=arrays(3, VC=(2, None))), "NULL")
        refused(call(of=arrays(3, KS=(1, 4104))), "16-byte")
    refused(commit(seqs=-1), "seqs")
    refused(commit(width=65), "width")
    refused(commit(table=NULL), "NULL")
    refused(commit(path=NULL), "NULL")
    refused(commit(ldt=3), "table")
    refused(commit(tw=0), "table")
    refused(commit(context=ctypes.c_void_p(4098)), "aligned")
    refused(copy(count=-1), "count")
    refused(copy(copies=NULL), "NULL")
    refused(copy(copies=ctypes.c_void_p(4098)), "aligned")
    assert commit(seqs=0) == 0 and copy(count=0) == 0


def test_update_refusals(lib):
    size = lib.gptq2d_pages_update_workspace_size
    assert size(0, 5) == 0 and size(5, 0) == 0 and size(5, 100) > 0
    ok = dict(rows=2, old=3, tw=4, table=P, ldt=4, length=P, source=P, want=P, held=P, pages=10, page=16,
              out=ctypes.c_void_p(8192), ldo=4, copies=P, left=P, ws=P, nb=size(2, 10), stream=None)
    call = lambda **k: lib.gptq2d_pages_update(*{**ok, **k}.values())
    refused(call(rows=0), "rows")
    refused(call(old=65536), "rows")
    refused(call(page=24), "page_size")
    refused(call(pages=0), "tokens")
    refused(call(pages=2 ** 31 // 16), "tokens")
    refused(call(tw=0), "table")
    refused(call(ldt=3), "table")
    refused(call(ldo=3), "table")
    refused(call(rows=65535, tw=65536, ldt=65536, ldo=65536), "2^31")
    for name in ("table", "length", "want", "out", "copies"):
        refused(call(**{name: NULL}), "NULL")
    refused(call(rows=4, source=NULL), "sources")
    refused(call(left=ctypes.c_void_p(4098)), "aligned")
    refused(call(out=P), "share memory")
    refused(call(out=ctypes.c_void_p(4096 + 4 * 11)), "share memory")
    assert call(nb=ok["nb"] - 1) == -6 and call(ws=ctypes.c_void_p(4100)) == -6


def test_binding_checks():
    t = torch.zeros(2, 3)
    with pytest.raises(ValueError, match="device tensor"):
        binding.gptq2d_tree_verify(t, torch.zeros(1, 2, dtype=torch.long), None, None, 1.0, None, None, None, 1.0, *[None] * 5)
    with pytest.raises(ValueError, match="no layer"):
        binding.gptq2d_cache_copy([], torch.zeros(1, 3, dtype=torch.int32))
    with pytest.raises(TypeError, match="int32"):
        binding.gptq2d_pages_update(torch.zeros(2, 3), torch.zeros(2), None, torch.zeros(2), None, 5, 16, t, None, None, None)


@pytest.mark.parametrize("seed", range(8))
def test_oracle_of_page_tables(seed):
    """No page is written that another row, or somebody else, reads."""
    rng = random.Random(seed)
    page, width, rows = 16, 6, 9
    pages = 80
    names = rng.sample(range(pages), rows * width)
    table = [names[i * width:(i + 1) * width] for i in range(rows)]
    length = [rng.randint(0, width * page) for _ in range(rows)]
    held = [int(rng.random() < 0.2) for _ in range(pages)]
    for _ in range(4):
        source = [rng.randint(-1, rows - 1) for _ in range(rows)]
        kept = [rng.randint(0, length[s]) if s >= 0 else 0 for s in source]
        want = [min(k + rng.randint(0, 20), width * page) for k in kept]
        kept = [min(length[s], w) if s >= 0 else 0 for s, w in zip(source, want)]
        out, copies, left = serving.pages_update(table, length, source, want, held, pages, page)
        for i in range(rows):
            for j in range(-(-want[i] // page)):
                if (j + 1) * page > kept[i]:  # the row writes here
                    p = out[i][j]
                    assert p < 0 or sum(r.count(p) for r in out) == 1 and not held[p]
            for j in range(kept[i] // page):
                assert out[i][j] == table[source[i]][j]
        used = {p for r in out for p in r if p >= 0}
        assert left < 0 or left == sum(p not in used and not held[p] for p in range(pages))
        assert not {c[1] for c in copies if c[1] >= 0} & {c[0] for c in copies if c[0] >= 0}
        table, length = out, want


def test_adapters_refusals(lib):
    size, back = lib.gptq2d_adapters_workspace_size, lib.gptq2d_adapters_backward_workspace_size
    assert size(0, 8, 8, 4, 2) == 0 and size(8, 8, 8, 129, 2) == 0 and size(8, 8, 8, 4, 2) > 0
    assert back(0, 8, 8, 4, 2) == 0 and back(8, 8, 8, 4, 5000) == 0 and back(8, 8, 8, 4, 2) > 0
    assert lib.gptq2d_adapter_groups_size(7, 3) == 19 and lib.gptq2d_adapter_groups_size(-1, 3) == 0
    refused(lib.gptq2d_adapter_groups(-1, 3, P, P, None), "M")
    refused(lib.gptq2d_adapter_groups(5, 0, P, P, None), "count")
    refused(lib.gptq2d_adapter_groups(2 ** 22, 2048, P, P, None), "2^32")
    refused(lib.gptq2d_adapter_groups(5, 3, NULL, P, None), "NULL")
    refused(lib.gptq2d_adapter_groups(5, 3, P, ctypes.c_void_p(4098), None), "aligned")
    shape = dict(M=8, N=16, K=24, R=4, count=2, dt=BF16)
    ok = dict(**shape, X=P, ldx=24, A=P, lda=24, B=P, ldb=4, scales=P, groups=P, Y=P, ldy=16, O=P, ldo=16, H=P, ws=P,
              nb=size(8, 16, 24, 4, 2), stream=None)
    call = lambda **k: lib.gptq2d_adapters(*{**ok, **k}.values())
    for k in (dict(M=-1), dict(M=2 ** 22 + 1), dict(N=0), dict(K=2 ** 22 + 1)):
        refused(call(**k), "M, N and K")
    refused(call(R=0), "R in")
    refused(call(R=129), "R in")
    refused(call(count=4097), "count")
    refused(call(dt=F64), "dtype")
    for name in ("X", "A", "B", "groups", "O"):
        refused(call(**{name: NULL}), "NULL")
    for name in ("ldx", "lda", "ldb", "ldy", "ldo"):
        refused(call(**{name: ok[name] - 1}), "leading dimension")
    refused(call(Y=ctypes.c_void_p(4097)), "aligned")
    refused(call(H=ctypes.c_void_p(4098)), "aligned")
    assert call(M=0) == 0  # no work
    assert call(nb=ok["nb"] - 1) == -6 and call(ws=ctypes.c_void_p(4100)) == -6
    ok = dict(**shape, G=P, ldg=16, X=P, ldx=24, A=P, lda=24, B=P, ldb=4, scales=P, groups=P, H=P, D=P, ldd=24, dX=P, lddx=24,
              dA=P, dB=P, ws=P, nb=back(8, 16, 24, 4, 2), stream=None)
    call = lambda **k: lib.gptq2d_adapters_backward(*{**ok, **k}.values())
    refused(call(R=129), "R in")
    refused(call(dt=F64), "dtype")
    refused(call(dX=NULL, dA=NULL, dB=NULL), "no gradient")
    refused(call(groups=NULL), "NULL")
    refused(call(G=NULL), "NULL")
    refused(call(A=NULL), "dX needs A")
    refused(call(B=NULL), "need B")
    refused(call(X=NULL), "dA needs X")
    refused(call(H=NULL), "dB needs H")
    for name in ("ldg", "ldx", "lda", "ldb", "ldd", "lddx"):
        refused(call(**{name: ok[name] - 1}), "leading dimension")
    refused(call(dX=ctypes.c_void_p(4097)), "aligned")
    refused(call(dB=ctypes.c_void_p(4098)), "aligned")
    assert call(nb=ok["nb"] - 1) == -6 and call(ws=NULL) == -6


def test_adapter_weights():
    """Adapters behind one another, with a row stride; other layouts are refused."""
    with pytest.raises(ValueError, match=r"\[count, R, K\]"):
        binding._adapter_weights(torch.zeros(2, 4, 8), torch.zeros(2, 8, 5), None)
    with pytest.raises(ValueError, match="behind one another"):
        binding._adapter_weights(torch.zeros(3, 4, 8)[::2], torch.zeros(2, 8, 4), None)
    with pytest.raises(ValueError, match="device tensor"):
        binding._adapter_weights(torch.zeros(2, 4, 8), torch.zeros(2, 8, 4), None)


def test_adapter_sizes(lib):
    """Batches whose work groups would be too many are refused, and have no workspace."""
    args = lambda M, N, K: (M, N, K, 4, 2, binding.BF16, P, K, P, K, P, 4, NULL, P, NULL, N, P, N, NULL, P, 1 << 60, None)
    back = lambda M, N, K: (M, N, K, 4, 2, binding.BF16, P, N, P, K, P, K, P, 4, NULL, P, P, NULL, K, P, K, P, P, P, 1 << 60, None)
    for M, N, K in ((1 << 20, 1 << 18, 8), (1 << 20, 8, 1 << 18), (1 << 22, 8, (1 << 15) + 1)):
        refused(lib.gptq2d_adapters(*args(M, N, K)), "2^37")
        refused(lib.gptq2d_adapters_backward(*back(M, N, K)), "2^37")
        assert lib.gptq2d_adapters_workspace_size(M, N, K, 4, 2) == 0
        assert lib.gptq2d_adapters_backward_workspace_size(M, N, K, 4, 2) == 0
    assert lib.gptq2d_adapters_workspace_size(1 << 22, 8, 1 << 15, 4, 2) > 0


def test_gradients_of_no_rows(lib):
    """An empty batch's tensors have no memory: a dX of no rows is nothing to do, not nothing asked for."""
    args = lambda M, dX: (M, 16, 24, 4, 2, BF16, NULL, 16, NULL, 24, P, 24, P, 4, P, P, NULL, NULL, 0, dX, 24, NULL, NULL, NULL,
                          0, None)
    assert lib.gptq2d_adapters_backward(*args(0, NULL)) == 0
    assert lib.gptq2d_adapters_backward(*args(0, P)) == 0
    refused(lib.gptq2d_adapters_backward(*args(8, NULL)), "no gradient")


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", range(5))
def test_adapters_refuse_tangents(which, grad):
    """No derivative is lost without a word: there is no forward-mode one."""
    tensors = [torch.zeros(5, 8), torch.zeros(2, 4, 8), torch.zeros(2, 6, 4), torch.zeros(5, 6), torch.ones(2)]
    with torch.autograd.forward_ad.dual_level(), torch.set_grad_enabled(grad):
        tensors[which] = torch.autograd.forward_ad.make_dual(tensors[which], torch.ones_like(tensors[which]))
        X, A, B, Y, scales = tensors
        with pytest.raises(NotImplementedError, match="tangents"):
            binding.adapters(X, A, B, None, Y, scales)
