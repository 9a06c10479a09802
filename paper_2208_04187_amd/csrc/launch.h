// Included inside the unnamed namespaces of the operators of a token model's layers: what their hosts' sides check and return.

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
size_t size_of(division_dtype dt) { return dt == DIVISION_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)
