/* tests/fake_hip.c with more than one device: memory belongs to the device
 * that was current when it was allocated, a stream to the one in its handle
 * (0x1000 + device). */
#define hipGetDevice one_device
#define hipMalloc plain_malloc
#include "fake_hip.c"
#undef hipGetDevice
#undef hipMalloc

int hipGetDeviceCount(int* count) { *count = 2; return OK; }

static int current;
void fake_set_device(int device) { current = device; }
int hipGetDevice(int* device) { *device = current; return OK; }

static struct { uintptr_t base; int device; } owners[MAX_RANGES];
static int n_owners;

int hipMalloc(void** p, size_t size)
{
    const int e = plain_malloc(p, size);
    if (e == OK && n_owners < MAX_RANGES) {
        owners[n_owners].base = (uintptr_t)*p;
        owners[n_owners++].device = current;
    }
    return e;
}

int hipPointerGetAttribute(void* data, int attribute, void* p)
{
    void* base;
    size_t size;
    (void)attribute;            /* the device's ordinal is the one that is asked for */
    if (hipMemGetAddressRange(&base, &size, p) != OK)
        return fail(INVALID_VALUE);
    for (int k = 0; k < n_owners; ++k)
        if (owners[k].base == (uintptr_t)base)
            *(int*)data = owners[k].device;
    return OK;
}

int hipStreamGetDevice(void* stream, int* device)
{
    *device = (int)((uintptr_t)stream - 0x1000);
    return OK;
}
