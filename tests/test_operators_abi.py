"""CPU checks of the eight-bit operators' C entry points: arguments are refused
with a status and a message before any device is touched, workspace sizes and
the binding's view checks."""
import ctypes

import pytest
import torch

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


def test_block_quantize_refusals(lib):
    ok = dict(rows=4, cols=40, dt=BF16, X=P, ldx=40, block_rows=1, pow2=0, Q=P, ldq=48, S=P, lds=4, QT=NULL, ldqt=0,
              ST=NULL, ldst=0, stream=None)
    call = lambda **k: lib.gptq2d_block_quantize(*{**ok, **k}.values())
    refused(call(rows=0), "[1, 2^22]")
    refused(call(cols=2 ** 22 + 1), "[1, 2^22]")
    refused(call(dt=F64), "dtype")
    refused(call(block_rows=64), "block_rows")
    refused(call(X=NULL), "X is NULL")
    refused(call(ldx=39), "leading dimension")
    refused(call(X=ctypes.c_void_p(4097)), "aligned")
    refused(call(Q=NULL), "neither")
    refused(call(S=NULL), "codes or scales")
    refused(call(ldq=40), "16-byte")
    refused(call(Q=ctypes.c_void_p(4104)), "16-byte")
    refused(call(ldq=32), "too small")
    refused(call(lds=3), "scales")
    refused(call(QT=P), "codes or scales")
    refused(call(QT=P, ST=P, ldqt=16, ldst=39), "scales")


def test_block_matmul_refusals(lib):
    ok = dict(M=100, N=200, K=300, A=P, lda=304, SA=P, ldsa=100, B=P, ldb=304, SB=P, ldsb=3, br=128, dt=F32, C=P,
              ldc=200, ws=NULL, nb=0, stream=None)
    call = lambda **k: lib.gptq2d_block_matmul(*{**ok, **k}.values())
    refused(call(K=0), "M, N and K")
    refused(call(M=2 ** 22, N=2 ** 22), "2^37")
    refused(call(br=2), "block_rows")
    refused(call(dt=7), "dtype")
    refused(call(ldsa=99), "scales")
    refused(call(ldsb=2), "scales")
    refused(call(br=1, ldsb=199), "scales")
    refused(call(lda=296), "16-byte")
    refused(call(ldc=199), "leading dimension")
    refused(call(C=NULL), "C is NULL")
    big = dict(M=100, N=200, K=30000, lda=30000, ldb=30000, ldsb=235)
    assert lib.gptq2d_block_matmul_workspace_size(100, 200, 30000) > 0
    assert call(**big) == -6 and "workspace" in binding.gptq2d_last_error()
    assert call(**big, ws=ctypes.c_void_p(4100), nb=1 << 30) == -6 and "256-byte" in binding.gptq2d_last_error()


def test_block_linear_refusals(lib):
    ws = lib.gptq2d_block_linear_workspace_size(10, 20, 30)
    assert ws > 0 and lib.gptq2d_block_linear_workspace_size(0, 20, 30) == 0
    ok = dict(M=10, N=20, K=30, dt=BF16, X=P, ldx=30, W=P, ldw=32, SW=P, ldsw=1, pow2=0, Y=P, ldy=20, ws=P, nb=ws,
              stream=None)
    call = lambda **k: lib.gptq2d_block_linear(*{**ok, **k}.values())
    refused(call(dt=F64), "dtype")
    refused(call(X=NULL), "X is NULL")
    refused(call(ldw=30), "16-byte")
    refused(call(Y=NULL), "Y is NULL")
    assert call(nb=ws - 1) == -6 and call(ws=NULL) == -6
    ws = lib.gptq2d_block_linear_backward_workspace_size(10, 20, 30)
    ok = dict(M=10, N=20, K=30, dt=BF16, dY=P, lddy=20, X=P, ldx=30, WT=P, ldwt=32, SWT=P, ldswt=1, pow2=0, dX=P,
              lddx=30, dW=P, lddw=30, ws=P, nb=ws, stream=None)
    call = lambda **k: lib.gptq2d_block_linear_backward(*{**ok, **k}.values())
    refused(call(dX=NULL, dW=NULL), "neither")
    refused(call(dY=NULL), "dY is NULL")
    refused(call(X=NULL), "X is NULL")
    refused(call(WT=NULL), "codes or scales")
    refused(call(lddw=29), "leading dimension")
    assert call(nb=ws - 1) == -6


def test_cache_refusals(lib):
    ok = dict(tokens=5, heads=2, dim=64, dt=BF16, K=P, ldk=128, V=P, ldv=128, slots=P, code=0, pages=4, page=16, KC=P,
              VC=P, KS=P, VS=P, stream=None)
    call = lambda **k: lib.gptq2d_cache_append(*{**ok, **k}.values())
    refused(call(heads=0), "heads")
    refused(call(dim=24), "dim")
    refused(call(dim=272), "dim")
    refused(call(code=2), "code")
    refused(call(page=24), "page_size")
    refused(call(page=8192), "page_size")
    refused(call(pages=0), "tokens")
    refused(call(pages=2 ** 31 // 16), "tokens")
    refused(call(KC=NULL), "NULL")
    refused(call(VS=ctypes.c_void_p(4104)), "16-byte")
    refused(call(tokens=-1), "tokens")
    refused(call(dt=F64), "dtype")
    refused(call(K=NULL), "NULL")
    refused(call(ldv=127), "leading dimension")
    refused(call(slots=ctypes.c_void_p(4100)), "aligned")
    assert call(tokens=0) == 0  # no work
    ok = dict(tokens=5, heads=2, dim=64, dt=BF16, slots=P, code=0, pages=4, page=16, KC=P, VC=P, KS=P, VS=P, K=P,
              ldk=128, V=P, ldv=120, stream=None)
    refused(lib.gptq2d_cache_read(*ok.values()), "leading dimension")


def test_tree_refusals(lib):
    refused(lib.gptq2d_tree_masks(2, 65, P, P, None), "width")
    refused(lib.gptq2d_tree_masks(-1, 3, P, P, None), "seqs")
    refused(lib.gptq2d_tree_masks(2, 3, NULL, P, None), "NULL")
    assert lib.gptq2d_tree_masks(0, 3, NULL, NULL, None) == 0
    size = lib.gptq2d_tree_attention_workspace_size
    assert size(2, 65, 4, 2, 64) == 0 and size(2, 4, 5, 2, 64) == 0 and size(1, 1, 32, 8, 128) > 0
    ok = dict(seqs=2, width=3, heads=4, kv=2, dim=64, dt=BF16, Q=P, ldq=256, code=0, pages=4, page=16, KC=P, VC=P, KS=P,
              VS=P, table=P, ldt=4, tw=4, context=P, drafts=NULL, masks=NULL, scale=0.1, O=P, ldo=256, lse=NULL, ws=P,
              nb=1 << 30, stream=None)
    call = lambda **k: lib.gptq2d_tree_attention(*{**ok, **k}.values())
    refused(call(seqs=0), "bad shape")
    refused(call(width=65), "bad shape")
    refused(call(heads=5), "bad shape")
    refused(call(seqs=65535, heads=256, ldq=16384, ldo=16384), "bad shape")
    refused(call(dt=F64), "dtype")
    refused(call(page=20), "page_size")
    refused(call(Q=NULL), "NULL")
    refused(call(context=NULL), "NULL")
    refused(call(ldq=255), "leading dimension")
    refused(call(ldt=3), "table")
    refused(call(tw=0), "table")
    refused(call(tw=2 ** 25, ldt=2 ** 25), "table")
    refused(call(scale=float("inf")), "scale")
    refused(call(masks=ctypes.c_void_p(4100)), "aligned")
    assert call(nb=10) == -6 and call(ws=ctypes.c_void_p(4100)) == -6


def test_score_refusals(lib):
    assert lib.gptq2d_token_logprobs_workspace_size(1, 100000, 5) > 0
    assert lib.gptq2d_token_logprobs_workspace_size(1, 100000, 65) == 0
    ok = dict(rows=2, vocab=1000, dt=BF16, X=P, ldx=1000, scale=1.0, target=P, top=3, lp=P, H=P, lse=P, ids=P, tops=P,
              ws=NULL, nb=0, stream=None)
    call = lambda **k: lib.gptq2d_token_logprobs(*{**ok, **k}.values())
    refused(call(rows=2 ** 22 + 1), "rows")
    refused(call(vocab=0), "vocab")
    refused(call(top=65), "top")
    refused(call(vocab=2), "top")
    refused(call(dt=F64), "dtype")
    for s in (0.0, -1.0, float("nan"), float("inf")):
        refused(call(scale=s), "scale")
    refused(call(lse=NULL), "NULL")
    refused(call(ids=NULL), "NULL")
    refused(call(ldx=999), "leading dimension")
    refused(call(target=ctypes.c_void_p(4100)), "aligned")
    assert call(rows=0) == 0
    assert call(vocab=100000, ldx=100000) == -6
    ok = dict(rows=2, vocab=1000, dt=BF16, X=P, ldx=1000, scale=1.0, target=P, lse=P, H=P, gl=P, gh=P, dX=P, ldd=1000,
              stream=None)
    call = lambda **k: lib.gptq2d_token_logprobs_backward(*{**ok, **k}.values())
    refused(call(gl=NULL, gh=NULL), "no gradient")
    refused(call(target=NULL), "targets")
    refused(call(H=NULL), "entropy")
    refused(call(ldd=999), "leading dimension")
    refused(call(dX=NULL), "NULL")


def test_every_entry_point_is_bound(lib):
    for name in binding.declared_functions():
        assert hasattr(binding, name), name
        assert getattr(lib, name).argtypes is not None, name


def test_views_of_codes():
    """Codes need 16-byte rows that reach to a multiple of 16 columns; the check
    is the binding's (host tensors are refused first)."""
    buf = torch.zeros(4, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="device tensor"):
        binding._codes(buf, 4, 64, "Q")
    with pytest.raises(TypeError, match="float8"):
        binding._codes(buf.view(torch.uint8), 4, 64, "Q")
    with pytest.raises(TypeError, match="one dtype"):
        binding._narrow(torch.zeros(1), torch.zeros(1, dtype=torch.float16))
    with pytest.raises(TypeError, match="one dtype"):
        binding._narrow(torch.zeros(1, dtype=torch.float64))
